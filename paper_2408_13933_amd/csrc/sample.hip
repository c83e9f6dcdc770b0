// Drawing the next token of every row from its logits: temperature, the k
// most likely, the smallest set of a probability mass, a probability floor.
//
// Weights are integers, w = rint(2^40 exp((x - max x) / temperature)), so a
// sum is the same in whatever order it is made.  Logits are compared as
// 32-bit keys that ascend with them (0: never drawn).  The kept words are a
// prefix of the order (key descending, index ascending) in every setting: a
// cut is the last kept word's key and index.
//
// 1. scan: a wave reads 2048 logits, notes the largest and lists the few words
//    at or above a bound that 24 of its lanes' maxima reach.  Together the
//    lists hold every word of the row above the largest of these bounds.
// 2. sums (rows without top_k): the weights of all words, added per 2048 words
//    or, for top_p, per bin of logit distance from the largest.
// 3. gather (top_p rows whose cut is below what the lists hold): the words of
//    the cut's bin, and the weights above it per 2048 words.
// 4. draw: a block per row finds the cut among the listed or gathered words, by
//    bins of logit distance or, where too many of the listed share one, by the
//    bits of their keys, then the word; rows that neither serves (a top_k
//    larger than the lists hold, thousands of equal logits at the cut) walk
//    over the whole row by key bits.
//
// One reading of the logits bounds many rows, and the vector arithmetic of
// the weights (25 instructions each, fp64) those that need them all; one row
// is four launches, each its own latency.  us: 512 rows of 256000 fp32, settings
// mixed, 98 + 36 + 34 + 24 (the scan 5.4 TB/s, all 2.7); 48 rows of 32000
// codes, top_p, 5.2 + 8.0 + 7.4 + 10.0; one row of 256000, top_k, 5.2 + 1.8 + 1.8
// + 10.7.  Rows of top_p over flat logits, 512 of 256000: 160 + 190 for the
// second and third.  top_k = 300 of flat rows, per call: 1 row of 100000 28, 256
// rows of 256000 82 (over the whole row instead of the lists 330 and 1510).  A
// walk over the whole row, 1000 codes over words masked with the lowest: 1 row
// of 32000 170 to 180, 64 of 256000 1400 to 1540.
#include <algorithm>

#include "codes.h"
#include "sample.h"
#include "wave.h"

namespace mq {
namespace {

constexpr int kSeg = 2048;       // words of a list and of a sum
constexpr int kUnit = 512;       // words that a wave of the second and third kernel takes at once
constexpr int kList = 64;        // places in a wave's list
constexpr int kRank = 24;        // lane maxima at or above a list's bound
constexpr int kBins = 1024;
constexpr double kBinScale = 24.0;  // bins per factor of two: weights past the last are 0
constexpr int kDrawThreads = 512, kDrawWaves = kDrawThreads / 64;
constexpr int kEntries = 4096;   // listed words that the draw takes into LDS
constexpr int kGather = 2048;    // gathered words of a row
constexpr int kNear = 512;       // words of the cut's bin among the listed ones
constexpr double kOne = 1099511627776.0;  // 2^40

// A row's part of the workspace beyond its segments'.
struct RowWork {
    unsigned long long mass[kBins];
    uint32_t count[kBins];
    uint2 near[kGather];  // key, index of the words in the cut's bin
    uint32_t found;       // how many there are (also past the places)
    uint32_t pad[3];
};

struct SampleArgs {
    const void* x;
    int64_t ld;
    int32_t V, segs;
    double alpha;           // of 16-bit codes, whose zero-point drops out of all distances
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int32_t* tokens;
    uint4* info;            // [rows][segs]: largest key, bound, listed words
    uint2* list;            // [rows][segs][kList]: key, index
    int64_t* sums;          // [rows][segs]
    RowWork* work;          // [rows]
};

// Logits as they are compared: of_key(key(v)) == v for the values that occur.
struct Fp32 {
    using T = float;
    using V = float;
    static constexpr int kTopBit = 31;
    static constexpr uint32_t kLeast = 0x00800000u;  // of the least finite value
    static __device__ V load(float x) { return fmaxf(x, -__builtin_inff()); }  // no NaN
    static __device__ V none() { return -__builtin_inff(); }
    static __device__ V larger(V a, V b) { return fmaxf(a, b); }
    static __device__ uint32_t key(V x)
    {
        const uint32_t b = __float_as_uint(x + 0.0f);  // -0 is 0
        const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
        return x > -__builtin_inff() ? k : 0;  // NaN and -infinity are never drawn
    }
    static __device__ V of_key(uint32_t k)
    {
        return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
    }
};
struct Code16 {
    using T = int16_t;
    using V = int32_t;
    static constexpr int kTopBit = 16;
    static constexpr uint32_t kLeast = 1;
    static __device__ V load(int16_t q) { return (int32_t)q + 32769; }
    static __device__ V none() { return 0; }
    static __device__ V larger(V a, V b) { return max(a, b); }
    static __device__ uint32_t key(V v) { return (uint32_t)v; }
    static __device__ V of_key(uint32_t k) { return (int32_t)k; }
};

// A row's settings.
struct Row {
    double scale;    // log2(e) / temperature
    double p;        // top_p (1: off)
    int64_t floor;   // least weight of the min_p rule
    int32_t k;       // top_k (0: off)
    uint32_t kmax;   // key of its largest logit
    double max;      // that logit (fp32)
    double step;     // distance of neighbouring codes (16 bits)
    template <class F>
    __device__ void set_max(const SampleArgs& a, uint32_t key)
    {
        kmax = key;
        max = (double)F::of_key(key);
        step = a.alpha * scale;
    }
};

__device__ inline Row row_of(const SampleArgs& a, int64_t m)
{
    Row r;
    const double t = a.temperature ? (double)a.temperature[m] : 1.0;
    const int32_t k = a.top_k ? a.top_k[m] : 0;
    r.k = k > 0 && k < a.V ? k : 0;
    r.p = a.top_p ? (double)a.top_p[m] : 1.0;
    r.p = r.p < 1.0 ? fmax(r.p, 0.0) : 1.0;  // NaN: off
    const double mp = a.min_p ? (double)a.min_p[m] : 0.0;
    r.floor = mp > 0.0 ? (int64_t)ceil(fmin(mp, 1.0) * kOne) : 0;
    // finite (t >= 2^-149); not 0 even for an infinite t, so that an infinite
    // distance stays one
    r.scale = fmax(1.4426950408889634 / t, 1e-300);
    if (!(t > 0.0)) {  // greedy: the first of the largest
        r.k = 1;
        r.scale = 1.4426950408889634;
    }
    return r;
}

// The distance of a logit from the row's largest, in factors of two of its
// weight, at most 100.  The same for equal logits, never less for smaller
// ones; 100 for -infinity, and next to +infinity for all but that.
__device__ inline double distance(const Row& r, float v)
{
    return fmin(fmax((r.max - (double)v) * r.scale, 0.0), 100.0);  // infinity - infinity: 0
}
__device__ inline double distance(const Row& r, int32_t v)
{
    return fmin((double)((int32_t)r.kmax - v) * r.step, 100.0);
}

// rint(2^40 2^-z): z to the next 1/64, 2^(j/64) from a table in LDS (2^40 of
// it in entry j), exp2_rest; the last product is added to 1.5 * 2^52, whose low
// bits are then the rounded weight.
__device__ inline void init_table(double* table)  // by the block, which waits afterwards
{
    if (threadIdx.x < 64) table[threadIdx.x] = kOne * exp2_poly((double)threadIdx.x / 64.0);
}
__device__ inline int64_t weight_at(const double* table, double z)
{
    const double t = kTableShift - z;
    const double f = (kTableShift - t) - z;
    const int32_t k = rint_low(t);
    const int64_t e = __double_as_longlong(table[k & 63]);
    const int32_t hi = (int32_t)(e >> 32) + ((k & ~63) << 14);  // the exponent, k / 64 lower
    const double w = __builtin_fma(
        exp2_rest(f), __longlong_as_double(((int64_t)hi << 32) | (uint32_t)e), kRintShift);
    return __double_as_longlong(w) - __double_as_longlong(kRintShift);
}
template <class F>
__device__ inline int64_t weight(const Row& r, const double* table, uint32_t k)
{
    return k ? weight_at(table, distance(r, F::of_key(k))) : 0;
}

// The bin of a distance.
__device__ inline int32_t bin_at(double z) { return min((int32_t)(z * kBinScale), kBins - 1); }
template <class F>
__device__ inline int32_t bin_of(const Row& r, uint32_t k)
{
    return bin_at(distance(r, F::of_key(k)));
}

// Rows without top_k need the weights of all words, with top_p per bin; so do
// rows whose top_k is more than the lists are likely to hold (a list has at
// least 24 words, some of them below the largest bound).
__device__ inline bool needs_bins(const SampleArgs& a, const Row& r)
{
    return r.k == 0 ? r.p < 1.0 : r.k > 12 * a.segs + 12;
}
__device__ inline bool needs_sums(const SampleArgs& a, const Row& r)
{
    return r.k == 0 || needs_bins(a, r);
}

// Words i0, i0 + 64, ... of a row, `none` past its end; first: the least of
// them over the wave.  All loads are under way before the first is looked at.
template <class F, int N>
__device__ __forceinline__ void load_words(const SampleArgs& a, const typename F::T* x,
                                           int32_t first, int32_t i0, typename F::V (&v)[N])
{
    typename F::T t[N];
    if (first + 64 * N <= a.V) {
#pragma unroll
        for (int j = 0; j < N; ++j) t[j] = x[i0 + 64 * j];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = F::load(t[j]);
        return;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) t[j] = x[min(i0 + 64 * j, a.V - 1)];
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = i0 + 64 * j < a.V ? F::load(t[j]) : F::none();
}

template <class F>
__global__ __launch_bounds__(256) void sample_scan_kernel(SampleArgs a, int64_t row0)
{
    const int lane = threadIdx.x & 63;
    const int seg = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (seg >= a.segs) return;
    const int64_t m = blockIdx.y;
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + (row0 + m) * a.ld;
    const int32_t i0 = seg * kSeg + lane;
    typename F::V k[kSeg / 64];
    load_words<F>(a, x, seg * kSeg, i0, k);
    typename F::V most = F::none();
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) most = F::larger(most, k[j]);
    uint32_t top = F::key(most);
    // the largest bound of 16 leading bits that kRank lanes' maxima reach
    uint32_t bound = 0;
#pragma unroll
    for (int bit = F::kTopBit; bit > F::kTopBit - 16 && bit >= 0; --bit) {
        const uint32_t c = bound | (1u << bit);
        if (__popcll(__ballot(top >= c)) >= kRank) bound = c;
    }
    bound = max(bound, F::kLeast);
    typename F::V at_least = F::of_key(bound);
    int n = 0;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) n += __popcll(__ballot(k[j] >= at_least));
    if (n > kList) {  // the smallest bound that leaves no more than the list holds
        uint32_t b = 0;
#pragma unroll 1
        for (int bit = F::kTopBit; bit >= 0; --bit) {
            const uint32_t c = b | (1u << bit);
            const typename F::V v = F::of_key(c);
            int cnt = 0;
            // (bounds that are no value: NaN above +infinity, none reach them;
            // below the least, all do)
#pragma unroll
            for (int j = 0; j < kSeg / 64; ++j) cnt += __popcll(__ballot(k[j] >= v));
            if (c < F::kLeast || cnt > kList) b = c;
        }
        bound = b + 1;  // b: the largest key that too many reach
        at_least = F::of_key(bound);
    }
    const int64_t at = m * a.segs + seg;
    uint2* list = a.list + at * kList;
    int pos = 0;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) {
        const uint64_t hit = __ballot(k[j] >= at_least);
        if (hit) {
            if (k[j] >= at_least)
                list[pos + __popcll(hit & below)] =
                    make_uint2(F::key(k[j]), (uint32_t)(i0 + 64 * j));
            pos += __popcll(hit);
        }
    }
    top = wave_max(top);
    if (lane == 0) {
        a.info[at] = make_uint4(top, bound, (uint32_t)pos, 0);
        a.sums[at] = 0;
    }
    // the row's bins and counter start at zero too (stores before the loads
    // would be waited for with them)
    RowWork& work = a.work[m];
    for (int i = seg * 64 + lane; i < kBins; i += a.segs * 64) {
        work.mass[i] = 0;
        work.count[i] = 0;
    }
    if (seg == 0 && lane == 0) work.found = 0;
}

// The row's largest key and the largest bound of its lists (every lane of the
// wave).
__device__ inline uint2 row_info(const SampleArgs& a, int64_t m)
{
    uint32_t top = 0, bound = 1;
    for (int i = threadIdx.x & 63; i < a.segs; i += 64) {
        const uint4 v = a.info[m * a.segs + i];
        top = max(top, v.x);
        bound = max(bound, v.y);
    }
    return make_uint2(wave_max(top), wave_max(bound));
}

// The sum of the values of the threads before this one, and of all.
template <int WAVES>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* total, int64_t* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t s = wave_scan(v);
    __syncthreads();
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    *total = all;
    return before + s - v;
}

// A wave takes `units` units of 512 words in a row.
template <class F>
__global__ __launch_bounds__(256) void sample_sums_kernel(SampleArgs a, int64_t row0, int units)
{
    __shared__ unsigned long long mass[kBins];
    __shared__ uint32_t count[kBins];
    __shared__ double table[64];
    const int lane = threadIdx.x & 63;
    const int64_t m = blockIdx.y;
    Row r = row_of(a, row0 + m);
    if (!needs_sums(a, r)) return;
    const uint32_t kmax = row_info(a, m).x;
    if (kmax == 0) return;  // the same for the whole block
    r.set_max<F>(a, kmax);
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + (row0 + m) * a.ld;
    const int32_t first = (blockIdx.x * 4 + (threadIdx.x >> 6)) * units * kUnit;
    const bool bins = needs_bins(a, r);
    init_table(table);
    if (bins)
        for (int i = threadIdx.x; i < kBins; i += 256) {
            mass[i] = 0;
            count[i] = 0;
        }
    __syncthreads();
    typename F::V v[8], next[8];
    load_words<F>(a, x, first, first + lane, next);
#pragma unroll 1
    for (int n = 0; n < units; ++n) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = next[j];
        if (n + 1 < units)
            load_words<F>(a, x, first + (n + 1) * kUnit, first + (n + 1) * kUnit + lane, next);
        int64_t s = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double z = distance(r, v[j]);
            const int64_t w = v[j] != F::none() ? weight_at(table, z) : 0;
            if (bins) {
                if (w) {
                    const int32_t bin = bin_at(z);
                    atomicAdd(&mass[bin], (unsigned long long)w);
                    if (r.k) atomicAdd(&count[bin], 1u);
                }
            } else {
                s += w >= r.floor ? w : 0;
            }
        }
        if (bins) continue;
        s = wave_sum(s);
        const int32_t at = first + n * kUnit;
        if (lane == 0 && at < a.V)
            atomicAdd(reinterpret_cast<unsigned long long*>(&a.sums[m * a.segs + at / kSeg]),
                      (unsigned long long)s);
    }
    if (!bins) return;
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += 256) {
        if (mass[i]) atomicAdd(&a.work[m].mass[i], mass[i]);
        if (count[i]) atomicAdd(&a.work[m].count[i], count[i]);
    }
}

// What a search over bins finds: the first bin from the top that reaches the
// target (else the last one that holds anything), and the words and mass of
// the bins before it.
struct Found {
    int32_t bin;
    int64_t count, mass;
};

// Bins in LDS are kept so that the lanes that hold 16 neighbouring ones each
// read next to each other.
__device__ inline int32_t place_of(int32_t bin) { return (bin & 15) * 64 + (bin >> 4); }

// One wave looks for the bin; lane l holds bins 16 l on.  reaches(count,
// mass) of everything up to and with a bin.
template <class Reaches>
__device__ inline Found find_bin(const uint32_t* count, const unsigned long long* mass,
                                 Reaches reaches)
{
    static_assert(kBins == 64 * 16, "16 bins per lane");
    const int lane = threadIdx.x & 63;
    int64_t n = 0, w = 0;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        n += count[64 * i + lane];
        w += (int64_t)mass[64 * i + lane];
    }
    const int64_t ns = wave_scan(n), ws = wave_scan(w);
    Found f;
    // the first lane that reaches the target, or the last with anything; then
    // the same among its bins
    const uint64_t hit = __ballot(reaches(ns, ws)), some = __ballot(n > 0);
    const int l = hit ? __builtin_ctzll(hit) : some ? 63 - __builtin_clzll(some) : 0;
    const int64_t nb = wave_read(ns - n, l), mb = wave_read(ws - w, l);
    const int64_t c = lane < 16 ? count[64 * lane + l] : 0;
    const int64_t v = lane < 16 ? (int64_t)mass[64 * lane + l] : 0;
    const int64_t cs = wave_scan(c), vs = wave_scan(v);
    const uint64_t have = __ballot(c > 0), in = __ballot(c > 0 && reaches(nb + cs, mb + vs));
    const int i = in ? __builtin_ctzll(in) : have ? 63 - __builtin_clzll(have) : 0;
    f.bin = 16 * l + i;
    f.count = nb + wave_read(cs - c, i);
    f.mass = mb + wave_read(vs - v, i);
    return f;
}

// Where the cuts of a row lie in its bins.
struct Cuts {
    // top_k's cut is in bin k (kBins without top_k), after so many words and
    // so much mass
    int32_t k;
    int64_t k_count, k_mass;
    // top_p's is in one of bins [p0, p1], after that mass (without top_p the
    // bin of top_k's cut): the mass it is a part of is known up to the words
    // of bin k
    int32_t p0, p1;
    int64_t p_mass;
    double target;  // without top_k
};
struct CutLds {
    int64_t wave[16], k_count, k_mass, k_own, p_mass;
    int32_t k, p0, p1;
};
// Thread t of the block looks at kBins / THREADS bins.
template <int THREADS>
__device__ __forceinline__ Cuts find_cuts(const SampleArgs& a, const Row& r, int64_t m, CutLds& lds)
{
    constexpr int per = kBins / THREADS;
    const int b0 = threadIdx.x * per;
    int64_t w[per], s = 0, total;
#pragma unroll
    for (int i = 0; i < per; ++i) {
        w[i] = (int64_t)a.work[m].mass[b0 + i];
        s += w[i];
    }
    const int64_t before = block_scan<THREADS / 64>(s, &total, lds.wave);
    if (threadIdx.x == 0) {
        lds.k = kBins;
        lds.k_count = 0;
        lds.k_mass = total;
        lds.k_own = 0;
        lds.p0 = lds.p1 = kBins;
        lds.p_mass = total;
    }
    __syncthreads();
    if (r.k > 0) {
        int64_t c[per], n = 0, all;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            c[i] = a.work[m].count[b0 + i];
            n += c[i];
        }
        int64_t run = block_scan<THREADS / 64>(n, &all, lds.wave), mass = before;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            if (run < r.k && run + c[i] >= r.k) {
                lds.k = b0 + i;
                lds.k_count = run;
                lds.k_mass = mass;
                lds.k_own = w[i];
            }
            run += c[i];
            mass += w[i];
        }
        __syncthreads();
    }
    Cuts f{lds.k, lds.k_count, lds.k_mass, lds.k, lds.k, lds.k_mass, r.p * (double)total};
    if (r.p < 1.0) {
        // the first bins that reach the least and the most that top_p asks for
        const double least = r.p * (double)lds.k_mass;
        const double most = r.p * (double)(lds.k_mass + lds.k_own);
        int64_t run = before;
#pragma unroll
        for (int i = 0; i < per; ++i) {
            const bool first = b0 + i == 0;
            if (w[i] && (first || (double)run < least) && (double)(run + w[i]) >= least) {
                lds.p0 = b0 + i;
                lds.p_mass = run;
            }
            if (w[i] && (first || (double)run < most) && (double)(run + w[i]) >= most)
                lds.p1 = b0 + i;
            run += w[i];
        }
        __syncthreads();
        f.p0 = min(lds.p0, lds.k);
        f.p1 = min(lds.p1, lds.k);
        f.p_mass = lds.p0 <= lds.k ? lds.p_mass : lds.k_mass;
    }
    return f;
}

// Gathers the words of the cuts' bins and adds the weights above them.
template <class F>
__global__ __launch_bounds__(256) void sample_gather_kernel(SampleArgs a, int64_t row0, int units)
{
    __shared__ CutLds lds;
    __shared__ double table[64];
    const int lane = threadIdx.x & 63;
    const int64_t m = blockIdx.y;
    Row r = row_of(a, row0 + m);
    if (!needs_bins(a, r)) return;
    const uint2 info = row_info(a, m);
    if (info.x == 0) return;
    r.set_max<F>(a, info.x);
    init_table(table);
    const Cuts f = find_cuts<256>(a, r, m, lds);
    if (r.k == 0 && f.p1 < bin_of<F>(r, info.y)) return;  // the lists hold it
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + (row0 + m) * a.ld;
    const int32_t first = (blockIdx.x * 4 + (threadIdx.x >> 6)) * units * kUnit;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    RowWork& work = a.work[m];
    typename F::V v[8], next[8];
    load_words<F>(a, x, first, first + lane, next);
#pragma unroll 1
    for (int n = 0; n < units; ++n) {
        const int32_t i0 = first + n * kUnit;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = next[j];
        if (n + 1 < units) load_words<F>(a, x, i0 + kUnit, i0 + kUnit + lane, next);
        int64_t s = 0;
        uint32_t mine = 0;  // bit j: word j is in one of the bins
        int cnt = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const double z = distance(r, v[j]);
            const int32_t bin = v[j] != F::none() ? bin_at(z) : kBins + 1;
            if (bin < f.p0) {
                const int64_t w = weight_at(table, z);
                s += w >= r.floor ? w : 0;
            }
            const bool here = (bin >= f.p0 && bin <= f.p1) || bin == f.k;
            mine |= (uint32_t)here << j;
            cnt += __popcll(__ballot(here));
        }
        s = wave_sum(s);
        if (lane == 0 && s)
            atomicAdd(reinterpret_cast<unsigned long long*>(&a.sums[m * a.segs + i0 / kSeg]),
                      (unsigned long long)s);
        if (cnt == 0) continue;
        // places for all of the wave's at once
        uint32_t at = 0;
        if (lane == 0) at = atomicAdd(&work.found, (uint32_t)cnt);
        at = __shfl((int)at, 0);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint64_t hit = __ballot((mine >> j) & 1);
            const uint32_t to = at + __popcll(hit & below);
            if (((mine >> j) & 1) && to < kGather)
                work.near[to] = make_uint2(F::key(v[j]), (uint32_t)(i0 + 64 * j + lane));
            at += __popcll(hit);
        }
    }
}

// ---------------------------------------------------------------------------
// The draw.

struct DrawLds {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
    uint64_t word[kEntries];  // listed or gathered words, as order() has them
    uint64_t near[2 * kNear];
    uint32_t cursor[kBins];
    int64_t wave64[kDrawWaves];
    int32_t wave32[kDrawWaves];
    CutLds cuts;
    double table[64];
    uint32_t sel[4];
    int64_t sel64[4];
};

// A word as one number that ascends along the order.
__device__ __forceinline__ uint64_t order(uint32_t key, uint32_t idx)
{
    return ((uint64_t)~key << 32) | idx;
}
__device__ __forceinline__ uint32_t key_of(uint64_t w) { return ~(uint32_t)(w >> 32); }

// The last kept word.
struct Cut {
    uint32_t key, idx;
    int64_t mass;  // of it and all before it in the order
    __device__ bool keeps(uint32_t k, uint32_t i) const { return k > key || (k == key && i <= idx); }
};

// n words in LDS put in order (dst): each counts those before it, eight reads
// under way at once.
__device__ __forceinline__ void order_words(const uint64_t* src, int n, uint64_t* dst)
{
    for (int e = threadIdx.x; e < n; e += kDrawThreads) {
        const uint64_t w = src[e];
        int rank = 0, o = 0;
        for (; o + 8 <= n; o += 8) {
            uint64_t t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = src[o + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) rank += t[i] < w;
        }
        for (; o < n; ++o) rank += src[o] < w;
        dst[rank] = w;
    }
}

// The cut among n ordered words of one bin, by count (words of the bin kept)
// or by mass; before: the mass of the bins before.  Wave 0 looks, all get it.
template <class F, bool MASS>
__device__ __forceinline__ Cut cut_in_order(const Row& r, DrawLds& lds, const uint64_t* word,
                                            int n, int64_t before, int64_t keep, double target)
{
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        int64_t run = before;
        for (int e0 = 0; e0 < n; e0 += 64) {
            const uint64_t w = e0 + lane < n ? word[e0 + lane] : ~0ull;
            int64_t c = weight<F>(r, lds.table, key_of(w));
            c = wave_scan(c);
            // the last word is kept in any case that gets that far
            const bool here = MASS ? (double)(run + c) >= target : e0 + lane + 1 >= keep;
            const uint64_t hit = __ballot(e0 + lane < n && (here || e0 + lane == n - 1));
            if (hit) {
                if (lane == __builtin_ctzll(hit)) {
                    lds.sel[0] = key_of(w);
                    lds.sel[1] = (uint32_t)w;
                    lds.sel64[0] = run + c;
                }
                break;
            }
            run += wave_read(c, 63);
        }
    }
    __syncthreads();
    const Cut c{lds.sel[0], lds.sel[1], lds.sel64[0]};
    __syncthreads();
    return c;
}

// The words that a draw looks at: the listed ones in LDS or the whole row.
template <class F>
struct Words {
    const DrawLds* lds;
    const typename F::T* x;
    int32_t n;
    bool listed;
    __device__ uint32_t key(int32_t i) const
    {
        return listed ? key_of(lds->word[i]) : F::key(F::load(x[i]));
    }
    __device__ uint32_t index(int32_t i) const { return listed ? (uint32_t)lds->word[i] : (uint32_t)i; }
};

// The cut over the listed words in LDS by their bins (count and mass there
// already); false if its bin holds more words than there is room for.
template <class F, bool MASS>
__device__ __forceinline__ bool cut_listed(const Row& r, DrawLds& lds, int n, int64_t keep,
                                           double target, Cut& cut)
{
    if (threadIdx.x < 64) {
        const Found f = find_bin(lds.count, lds.mass, [=](int64_t c, int64_t w) {
            return MASS ? (double)w >= target : c >= keep;
        });
        if (threadIdx.x == 0) {
            lds.sel[0] = (uint32_t)f.bin;
            lds.sel[1] = 0;
            lds.sel64[0] = f.count;
            lds.sel64[1] = f.mass;
        }
    }
    __syncthreads();
    const int32_t bin = (int32_t)lds.sel[0];
    const int64_t count = lds.sel64[0], mass = lds.sel64[1];
    const int near = (int)lds.count[place_of(bin)];
    if (near > kNear) return false;
    for (int i = threadIdx.x; i < n; i += kDrawThreads)
        if (bin_of<F>(r, key_of(lds.word[i])) == bin)
            lds.near[atomicAdd(&lds.sel[1], 1u)] = lds.word[i];
    __syncthreads();
    order_words(lds.near, near, lds.near + kNear);
    cut = cut_in_order<F, MASS>(r, lds, lds.near + kNear, near, mass, keep - count, target);
    return true;
}

// The cut among n words in LDS that lie in bins [b0, b1], by finer bins; so
// many words and so much mass come before them.  False if too many share the
// finer bin.
template <class F, bool MASS>
__device__ __forceinline__ bool cut_gathered(const Row& r, DrawLds& lds, int n, int b0, int b1,
                                             int64_t count, int64_t mass, int64_t keep,
                                             double target, Cut& cut)
{
    const double fine = (double)kBins / (double)(b1 - b0 + 1);
    // -1: not one of them
    auto sub_bin = [&](uint32_t k) {
        const double z = distance(r, F::of_key(k));
        const int32_t b = bin_at(z);
        if (b < b0 || b > b1) return -1;
        return min(max((int32_t)((z * kBinScale - (double)b0) * fine), 0), kBins - 1);
    };
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kDrawThreads) {
        lds.count[i] = 0;
        lds.mass[i] = 0;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += kDrawThreads) {
        const uint32_t k = key_of(lds.word[i]);
        const int32_t b = sub_bin(k);
        if (b < 0) continue;
        atomicAdd(&lds.count[place_of(b)], 1u);
        atomicAdd(&lds.mass[place_of(b)], (unsigned long long)weight<F>(r, lds.table, k));
    }
    __syncthreads();
    if (threadIdx.x < 64) {
        const Found f = find_bin(lds.count, lds.mass, [=](int64_t c, int64_t w) {
            return MASS ? (double)(mass + w) >= target : count + c >= keep;
        });
        if (threadIdx.x == 0) {
            lds.sel[0] = (uint32_t)f.bin;
            lds.sel[1] = 0;
            lds.sel64[0] = count + f.count;
            lds.sel64[1] = mass + f.mass;
        }
    }
    __syncthreads();
    const int32_t bin = (int32_t)lds.sel[0];
    const int64_t c0 = lds.sel64[0], m0 = lds.sel64[1];
    const int near = (int)lds.count[place_of(bin)];
    if (near > kNear) return false;
    for (int i = threadIdx.x; i < n; i += kDrawThreads)
        if (sub_bin(key_of(lds.word[i])) == bin) lds.near[atomicAdd(&lds.sel[1], 1u)] = lds.word[i];
    __syncthreads();
    order_words(lds.near, near, lds.near + kNear);
    cut = cut_in_order<F, MASS>(r, lds, lds.near + kNear, near, m0, keep - c0, target);
    return true;
}

// The cut over all the words, bit by bit of the keys from the top: those that
// have the leading bits found so far are counted by the next ten.
template <class F, bool MASS>
__device__ __forceinline__ Cut cut_search(const Row& r, const Words<F>& ws, DrawLds& lds,
                                          int64_t count, double target)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t lo = 1, hi = r.kmax;
    int64_t n0 = 0, m0 = 0;  // words and mass above hi
    int64_t ties = 0;
    for (;;) {
        const uint32_t range = hi - lo;
        const int bits = range ? 32 - __builtin_clz(range) : 0;
        const int shift = bits > 10 ? bits - 10 : 0;
        __syncthreads();
        for (int i = tid; i < kBins; i += kDrawThreads) {
            lds.count[i] = 0;
            lds.mass[i] = 0;
        }
        __syncthreads();
        for (int i0 = tid; i0 < ws.n; i0 += 8 * kDrawThreads) {
            uint32_t k[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * kDrawThreads;
                k[u] = i < ws.n ? ws.key(i) : 0;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (k[u] < lo || k[u] > hi) continue;
                const int32_t at = place_of((int32_t)((hi - k[u]) >> shift));
                atomicAdd(&lds.count[at], 1u);
                atomicAdd(&lds.mass[at], (unsigned long long)weight<F>(r, lds.table, k[u]));
            }
        }
        __syncthreads();
        if (tid < 64) {
            const Found f = find_bin(lds.count, lds.mass, [=](int64_t c, int64_t w) {
                return MASS ? (double)(m0 + w) >= target : n0 + c >= count;
            });
            if (tid == 0) {
                lds.sel[0] = (uint32_t)f.bin;
                lds.sel64[0] = n0 + f.count;
                lds.sel64[1] = m0 + f.mass;
            }
        }
        __syncthreads();
        const uint32_t bin = lds.sel[0];
        n0 = lds.sel64[0];
        m0 = lds.sel64[1];
        hi = hi - (bin << shift);  // still >= lo: the bin holds a word
        const uint32_t span = (1u << shift) - 1;
        if (hi - lo > span) lo = hi - span;  // (keys of codes start at 1: hi - span may wrap)
        if (shift == 0) {
            ties = lds.count[place_of((int32_t)bin)];
            break;
        }
    }
    // the words at key lo: how many are kept, and which is the last
    const int64_t w = weight<F>(r, lds.table, lo);
    int64_t keep;
    if (MASS) {
        int64_t l = 1, h = ties;
        while (l < h) {
            const int64_t mid = (l + h) >> 1;
            if ((double)(m0 + mid * w) >= target) h = mid;
            else l = mid + 1;
        }
        keep = l;
    } else {
        keep = min(ties, count - n0);
    }
    const int32_t part = ((ws.n + kDrawWaves - 1) / kDrawWaves + 63) & ~63;
    const int32_t i0 = min(wave * part, ws.n), i1 = min(i0 + part, ws.n);
    int32_t t = 0;
    for (int32_t i = i0; i < i1; i += 64)
        t += __popcll(__ballot(i + lane < i1 && ws.key(i + lane) == lo));
    __syncthreads();
    if (lane == 0) lds.wave32[wave] = t;
    __syncthreads();
    int64_t seen = 0;
    for (int v = 0; v < wave; ++v) seen += lds.wave32[v];
    if (keep > seen && keep <= seen + t)
        for (int32_t i = i0; i < i1; i += 64) {
            const uint64_t tie = __ballot(i + lane < i1 && ws.key(i + lane) == lo);
            const int32_t c = __popcll(tie);
            if (keep <= seen + c) {
                const bool last = ((tie >> lane) & 1) &&
                                  seen + __popcll(tie & (((uint64_t)2 << lane) - 1)) == keep;
                if (last) lds.sel[1] = ws.index(i + lane);
                break;
            }
            seen += c;
        }
    __syncthreads();
    const Cut c{lo, lds.sel[1], m0 + keep * w};
    __syncthreads();
    return c;
}

// The word at which the running weight of the kept ones, in index order,
// passes u times their total; every wave walks a contiguous part.
template <class F>
__device__ __forceinline__ int32_t draw_word(const Row& r, const Words<F>& ws, DrawLds& lds,
                                             const Cut& cut, double u)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t part = ((ws.n + kDrawWaves - 1) / kDrawWaves + 63) & ~63;
    const int32_t i0 = min(wave * part, ws.n), i1 = min(i0 + part, ws.n);
    auto kept = [&](int32_t i) -> int64_t {
        if (i >= i1) return 0;
        const uint32_t k = ws.key(i);
        if (!cut.keeps(k, ws.index(i))) return 0;
        const int64_t w = weight<F>(r, lds.table, k);
        return w >= r.floor ? w : 0;
    };
    int64_t s = 0;
#pragma unroll 4
    for (int32_t i = i0; i < i1; i += 64) s += kept(i + lane);
    s = wave_sum(s);
    __syncthreads();
    if (lane == 0) lds.wave64[wave] = s;
    __syncthreads();
    int64_t total = 0, before = 0;
    for (int w = 0; w < kDrawWaves; ++w) {
        if (w < wave) before += lds.wave64[w];
        total += lds.wave64[w];
    }
    const int64_t target = min((int64_t)(u * (double)total), total - 1);
    if (threadIdx.x == 0) lds.sel[0] = 0;
    __syncthreads();
    if (target >= before && target < before + s) {
        int64_t run = before;
        for (int32_t i = i0; i < i1; i += 64) {
            int64_t c = kept(i + lane);
            c = wave_scan(c);
            const uint64_t hit = __ballot(run + c > target);
            if (hit) {
                if (lane == __builtin_ctzll(hit)) lds.sel[0] = ws.index(i + lane);
                break;
            }
            run += wave_read(c, 63);
        }
    }
    __syncthreads();
    return (int32_t)lds.sel[0];
}

// The word from the kept weights of every segment: sum(i) of segment i, the
// cut's own rule within the segment.
template <class F, class Sum>
__device__ __forceinline__ int32_t draw_by_segments(const SampleArgs& a, const Row& r, const typename F::T* x,
                                    DrawLds& lds, const Cut& cut, double u, Sum sum)
{
    const int tid = threadIdx.x;
    // neighbouring segments per thread
    const int each = (a.segs + kDrawThreads - 1) / kDrawThreads, first = tid * each;
    int64_t s = 0, total = 0;
    for (int i = first; i < min(first + each, a.segs); ++i) s += sum(i);
    int64_t run = block_scan<kDrawWaves>(s, &total, lds.wave64);
    const int64_t target = min((int64_t)(u * (double)total), total - 1);
    if (tid == 0) {
        lds.sel[0] = 0;
        lds.sel64[0] = 0;
    }
    __syncthreads();
    if (target >= run && target < run + s) {
        int i = first;
        for (int64_t v; target >= run + (v = sum(i)); ++i) run += v;
        lds.sel[0] = (uint32_t)i;
        lds.sel64[0] = run;
    }
    __syncthreads();
    // neighbouring words of that segment per thread
    constexpr int per = kSeg / kDrawThreads;
    const int32_t i0 = (int32_t)lds.sel[0] * kSeg + tid * per;
    run = lds.sel64[0];
    typename F::T v[per];
    int64_t w[per];
#pragma unroll
    for (int j = 0; j < per; ++j) v[j] = x[min(i0 + j, a.V - 1)];
    s = 0;
#pragma unroll
    for (int j = 0; j < per; ++j) {
        const uint32_t k = i0 + j < a.V ? F::key(F::load(v[j])) : 0;
        w[j] = cut.keeps(k, (uint32_t)(i0 + j)) ? weight<F>(r, lds.table, k) : 0;
        if (w[j] < r.floor) w[j] = 0;
        s += w[j];
    }
    int64_t all;
    run += block_scan<kDrawWaves>(s, &all, lds.wave64);
    if (target >= run && target < run + s) {
        int32_t at = i0;
#pragma unroll
        for (int j = 0; j < per; ++j) {
            at += target >= run + w[j];  // (not once it is reached: the rest adds to run)
            run += w[j];
        }
        lds.sel[0] = (uint32_t)at;
    }
    __syncthreads();
    return (int32_t)lds.sel[0];
}

// A wave's lists of one turn, all loads under way at once.
constexpr int kTurn = 16;
__device__ __forceinline__ int draw_wave()
{
    return __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
}
// Lanes below this one in a mask.
__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                          __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}
struct Lists {
    uint2 e[kTurn];
    uint32_t n;  // lane i: of list i (0 past the wave's)
    int lists;   // of this wave in the turn
    __device__ __forceinline__ void load(const SampleArgs& a, int64_t m, int s0)
    {
        // neighbouring lists, as many for each wave
        const int lane = threadIdx.x & 63, left = min(a.segs - s0, kTurn * kDrawWaves);
        const int each = (left + kDrawWaves - 1) / kDrawWaves, first = s0 + draw_wave() * each;
        lists = min(max(s0 + left - first, 0), each);
        const int64_t at = m * a.segs + min(first, a.segs - 1);
        n = lane < lists ? a.info[at + lane].z : 0;
        // (places past the list's words: anything)
#pragma unroll
        for (int i = 0; i < kTurn; ++i)
            if ((i & ~3) < lists) e[i] = a.list[(at + min(i, max(lists - 1, 0))) * kList + lane];
    }
};

// The listed words from the bound on into LDS, in index order; how many there
// are (more than kEntries: not all of them are there).  t: the first turn.
__device__ __forceinline__ int64_t store_lists(const SampleArgs& a, int64_t m, uint32_t bound,
                                               Lists& t, DrawLds& lds)
{
    const int lane = threadIdx.x & 63, wave = draw_wave();
    int64_t n = 0;
    for (int s0 = 0; s0 < a.segs; s0 += kTurn * kDrawWaves) {
        if (s0) t.load(a, m, s0);
        uint64_t hit[kTurn];
        int mine = 0;
#pragma unroll
        for (int i = 0; i < kTurn; ++i)
            if ((i & ~3) < t.lists) {  // (four at a time)
                hit[i] = __ballot(lane < __builtin_amdgcn_readlane((int)t.n, i) &&
                                  t.e[i].x >= bound);
                mine += __popcll(hit[i]);
            }
        __syncthreads();
        if (lane == 0) lds.wave32[wave] = mine;
        __syncthreads();
        int before = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kDrawWaves; ++w) {
            before += w < wave ? lds.wave32[w] : 0;
            all += lds.wave32[w];
        }
        // (places past the last: not stored; n stays below 2^22)
        int at = __builtin_amdgcn_readfirstlane((int)n + before);
#pragma unroll
        for (int i = 0; i < kTurn; ++i)
            if ((i & ~3) < t.lists) {
                const int to = at + lanes_below(hit[i]);
                if (((hit[i] >> lane) & 1) && to < kEntries)
                    lds.word[to] = order(t.e[i].x, t.e[i].y);
                at += __popcll(hit[i]);
            }
        n += all;
    }
    __syncthreads();
    return n;
}

// The draw from the `few` <= kDrawThreads listed words (n in LDS, in index
// order, counted by bin) of the bins up to `bin`, which hold the kept ones: a
// thread per word.  mass: top_p's, or negative: p of the sum of the first k.
//
// A word's place in the order is what the bins before its own hold and what
// comes before it in its own.
template <class F>
__device__ __forceinline__ int32_t draw_few(const Row& r, DrawLds& lds, int n, int32_t bin,
                                            int few, double mass, double u)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = draw_wave();
    // the words of these bins, in index order
    static_assert(kEntries / kDrawThreads <= 32, "a bit per turn");
    const int32_t part = ((n + kDrawWaves - 1) / kDrawWaves + 63) & ~63;
    const int32_t i0 = min(wave * part, n), i1 = min(i0 + part, n);
    uint32_t mine = 0;  // bit j: the lane's word of turn j is one of them
    int cnt = 0;
#pragma unroll 1
    for (int j = 0; i0 + 64 * j < i1; ++j) {
        const int32_t i = i0 + 64 * j + lane;
        const bool here = i < i1 && bin_of<F>(r, key_of(lds.word[min(i, n - 1)])) <= bin;
        mine |= (uint32_t)here << j;
        cnt += __popcll(__ballot(here));
    }
    // and the places of the bins
    const uint32_t c0 = lds.count[place_of(2 * tid)], c1 = lds.count[place_of(2 * tid + 1)];
    if (lane == 0) lds.wave32[wave] = cnt;
    int64_t total;
    const int64_t start = block_scan<kDrawWaves>((int64_t)(c0 + c1), &total, lds.wave64);
    lds.cursor[2 * tid] = (uint32_t)start;
    lds.cursor[2 * tid + 1] = (uint32_t)start + c0;
    int at = 0;
#pragma unroll
    for (int w = 0; w < kDrawWaves; ++w) at += w < wave ? lds.wave32[w] : 0;
#pragma unroll 1
    for (int j = 0; i0 + 64 * j < i1; ++j) {
        const bool here = (mine >> j) & 1;
        const uint64_t hit = __ballot(here);
        if (here) lds.near[at + lanes_below(hit)] = lds.word[i0 + 64 * j + lane];
        at += __popcll(hit);
    }
    __syncthreads();
    const bool have = tid < few;
    const uint64_t word = have ? lds.near[tid] : 0;
    const uint32_t key = key_of(word);
    const int32_t own = have ? bin_of<F>(r, key) : 0;
    if (have) lds.near[kNear + atomicAdd(&lds.cursor[own], 1u)] = word;
    __syncthreads();
    int rank = 0;
    if (have) {
        const int end = (int)lds.cursor[own];
        int o = end - (int)lds.count[place_of(own)];
        rank = o;
        for (; o + 8 <= end; o += 8) {
            uint64_t t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = lds.near[kNear + o + i];
#pragma unroll
            for (int i = 0; i < 8; ++i) rank += t[i] < word;
        }
        for (; o < end; ++o) rank += lds.near[kNear + o] < word;
    }
    const int64_t w = have && (r.k == 0 || rank < r.k) ? weight<F>(r, lds.table, key) : 0;
    // the weights before it in the order
    if (have) lds.mass[rank] = (unsigned long long)w;
    __syncthreads();
    const int64_t sorted = have ? (int64_t)lds.mass[tid] : 0;
    const int64_t ahead = block_scan<kDrawWaves>(sorted, &total, lds.wave64);
    if (have) lds.mass[tid] = (unsigned long long)ahead;
    __syncthreads();
    const int64_t before = have ? (int64_t)lds.mass[rank] : 0;
    if (mass < 0.0) mass = r.p * (double)total;
    const bool kept = (r.p >= 1.0 || rank == 0 || (double)before < mass) && w >= r.floor;
    const int64_t kw = have && kept ? w : 0;
    // the kept weights before it in index order
    const int64_t run = block_scan<kDrawWaves>(kw, &total, lds.wave64);
    const int64_t target = min((int64_t)(u * (double)total), total - 1);
    if (kw > 0 && target >= run && target < run + kw) lds.sel[0] = (uint32_t)word;
    __syncthreads();
    return (int32_t)lds.sel[0];
}

template <class F>
__global__ __launch_bounds__(kDrawThreads, 4) void sample_draw_kernel(SampleArgs a, int64_t row0)
{
    __shared__ DrawLds lds;
    const int tid = threadIdx.x;
    const int64_t m = blockIdx.x, row = row0 + m;
    Lists lists;  // under way from the start
    lists.load(a, m, 0);
    const uint2 info = row_info(a, m);
    Row r = row_of(a, row);
    const double u0 = (double)a.u[row], u = u0 > 0.0 ? fmin(u0, 1.0) : 0.0;
    const uint32_t bound = info.y;
    if (info.x == 0) {  // nothing can be drawn
        if (tid == 0) a.tokens[row] = -1;
        return;
    }
    r.set_max<F>(a, info.x);
    init_table(lds.table);
    __syncthreads();
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + row * a.ld;
    const int64_t* sums = a.sums + m * a.segs;
    const bool bins = needs_bins(a, r);

    if (needs_sums(a, r) && !bins) {  // no cut
        const Cut all{1, 0xffffffffu, 0};
        const int32_t tok = draw_by_segments<F>(a, r, x, lds, all, u, [&](int i) { return sums[i]; });
        if (tid == 0) a.tokens[row] = tok;
        return;
    }

    Cut cut{1, 0xffffffffu, 0};
    double target = 0.0;
    if (bins) {
        const Cuts f = find_cuts<kDrawThreads>(a, r, m, lds.cuts);
        target = f.target;
        const RowWork& work = a.work[m];
        const int n = (int)min(work.found, (uint32_t)0x7fffffff);
        const bool gathered = r.k > 0 || f.p1 >= bin_of<F>(r, bound);
        bool found = gathered && n <= kGather && a.segs <= kBins;
        if (found) {
            for (int i = tid; i < n; i += kDrawThreads)
                lds.word[i] = order(work.near[i].x, work.near[i].y);
            double mass = target;
            if (r.k > 0 && f.k == kBins) {  // fewer than k have a weight
                mass = r.p * (double)f.k_mass;
            } else if (r.k > 0) {
                found = cut_gathered<F, false>(r, lds, n, f.k, f.k, f.k_count, f.k_mass, r.k, 0.0,
                                               cut);
                mass = r.p * (double)cut.mass;
            }
            if (found && r.p < 1.0)
                found = cut_gathered<F, true>(r, lds, n, f.p0, f.p1, 0, f.p_mass, 0, mass, cut);
        }
        if (found) {
            // the segments' sums, which the kept ones of these words join
            __syncthreads();
            for (int i = tid; i < a.segs; i += kDrawThreads)
                lds.mass[i] = (unsigned long long)sums[i];
            __syncthreads();
            for (int i = tid; i < n; i += kDrawThreads) {
                const uint32_t k = key_of(lds.word[i]), at = (uint32_t)lds.word[i];
                if (!cut.keeps(k, at)) continue;
                const int64_t w = weight<F>(r, lds.table, k);
                if (w >= r.floor) atomicAdd(&lds.mass[at / kSeg], (unsigned long long)w);
            }
            __syncthreads();
            const int32_t tok = draw_by_segments<F>(a, r, x, lds, cut, u,
                                                    [&](int i) { return (int64_t)lds.mass[i]; });
            if (tid == 0) a.tokens[row] = tok;
            return;
        }
        cut = Cut{1, 0xffffffffu, 0};
        __syncthreads();
    }

    const int64_t n = store_lists(a, m, bound, lists, lds);
    bool listed = n > 0 && n <= kEntries && n >= r.k;
    if (listed) {
        for (int i = tid; i < kBins; i += kDrawThreads) {
            lds.count[i] = 0;
            lds.mass[i] = 0;
        }
        __syncthreads();
        int64_t s = 0, all;
        for (int i = tid; i < n; i += kDrawThreads) {
            const uint32_t k = key_of(lds.word[i]);
            const int32_t at = place_of(bin_of<F>(r, k));
            const int64_t w = weight<F>(r, lds.table, k);
            s += w;
            atomicAdd(&lds.count[at], 1u);
            atomicAdd(&lds.mass[at], (unsigned long long)w);
        }
        block_scan<kDrawWaves>(s, &all, lds.wave64);
        listed = r.k > 0 || (double)all >= target;
    }
    bool found = false;
    if (listed) {
        // the bin of top_k's cut, without top_k of top_p's
        if (tid < 64) {
            const Found f = find_bin(lds.count, lds.mass, [=](int64_t c, int64_t w) {
                return r.k > 0 ? c >= r.k : (double)w >= target;
            });
            if (tid == 0) {
                lds.sel[0] = (uint32_t)f.bin;
                lds.sel[1] = 0;
                lds.sel64[0] = f.count;
                lds.sel64[1] = f.mass;
            }
        }
        __syncthreads();
        const int32_t bin = (int32_t)lds.sel[0];
        const int64_t count = lds.sel64[0] + lds.count[place_of(bin)];
        if (count <= kNear) {
            const int32_t tok = draw_few<F>(r, lds, (int)n, bin, (int)count,
                                            r.k > 0 ? -1.0 : target, u);
            if (tid == 0) a.tokens[row] = tok;
            return;
        }
        __syncthreads();
        if (r.k > 0) {
            found = cut_listed<F, false>(r, lds, (int)n, r.k, 0.0, cut);
            if (found && r.p < 1.0)
                found = cut_listed<F, true>(r, lds, (int)n, 0, r.p * (double)cut.mass, cut);
        } else {
            found = cut_listed<F, true>(r, lds, (int)n, 0, target, cut);
        }
    }
    // the listed words hold the cut, in whichever way it is found
    const Words<F> ws{&lds, x, listed ? (int32_t)n : a.V, listed};
    if (!found) {
        if (r.k > 0) {
            cut = cut_search<F, false>(r, ws, lds, r.k, 0.0);
            target = r.p * (double)cut.mass;
        }
        if (r.p < 1.0) cut = cut_search<F, true>(r, ws, lds, 0, target);
    }
    const int32_t tok = draw_word<F>(r, ws, lds, cut, u);
    if (tid == 0) a.tokens[row] = tok;
}

int32_t segments(int64_t V) { return (int32_t)((V + kSeg - 1) / kSeg); }

// Bytes per row of the workspace: its segments', and its own.
int64_t row_bytes(int64_t V)
{
    return (int64_t)segments(V) * (16 + 8 * kList + 8) + 8 + (int64_t)sizeof(RowWork);
}

template <class F>
hipError_t launch(SampleArgs a, int64_t M, char* ws, int64_t ws_bytes, hipStream_t s)
{
    const int64_t rows = std::min<int64_t>(ws_bytes / row_bytes(a.V), 65535);
    for (int64_t m0 = 0; m0 < M; m0 += rows) {
        const int64_t n = std::min(rows, M - m0);
        a.work = reinterpret_cast<RowWork*>(ws);
        a.info = reinterpret_cast<uint4*>(ws + n * sizeof(RowWork));
        a.list = reinterpret_cast<uint2*>(ws + n * (sizeof(RowWork) + a.segs * 16));
        a.sums = reinterpret_cast<int64_t*>(ws + n * (sizeof(RowWork) + a.segs * (16 + 8 * kList)));
        const dim3 g((unsigned)((a.segs + 3) / 4), (unsigned)n);
        sample_scan_kernel<F><<<g, 256, 0, s>>>(a, m0);
        // a wave per segment where that fills the chip (each work-group adds its
        // bins to the row's), else per unit.  512 rows of 256000, a fifth of
        // them with sums: 4 units 37 us, 8 45, 16 62
        const int units = n * a.segs >= 8192 ? kSeg / kUnit : 1;
        const dim3 gu((unsigned)((a.V + 4 * units * kUnit - 1) / (4 * units * kUnit)), (unsigned)n);
        sample_sums_kernel<F><<<gu, 256, 0, s>>>(a, m0, units);
        if (a.top_p || a.top_k) sample_gather_kernel<F><<<gu, 256, 0, s>>>(a, m0, units);
        sample_draw_kernel<F><<<(unsigned)n, kDrawThreads, 0, s>>>(a, m0);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

int64_t sample_workspace(int64_t M, int64_t V, bool least)
{
    const int64_t one = row_bytes(V), most = 64 << 20;
    return least ? one : std::max(one, std::min(M * one, most));
}

hipError_t launch_sample(const void* x, int32_t bits, int64_t M, int64_t V, int64_t ld, float alpha,
                         const float* temperature, const int32_t* top_k, const float* top_p,
                         const float* min_p, const float* u, int32_t* tokens, void* ws,
                         int64_t ws_bytes, hipStream_t s)
{
    SampleArgs a;
    a.x = x;
    a.ld = ld;
    a.V = (int32_t)V;
    a.segs = segments(V);
    a.alpha = alpha;
    a.temperature = temperature;
    a.top_k = top_k;
    a.top_p = top_p;
    a.min_p = min_p;
    a.u = u;
    a.tokens = tokens;
    return bits == 32 ? launch<Fp32>(a, M, static_cast<char*>(ws), ws_bytes, s)
                      : launch<Code16>(a, M, static_cast<char*>(ws), ws_bytes, s);
}

}  // namespace mq
