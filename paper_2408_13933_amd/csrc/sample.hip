// Drawing the next token of every row from its logits: temperature, the k
// most likely, the smallest set of a probability mass, a probability floor.
//
// Weights are integers, w = rint(2^40 exp((x - max x) / temperature)), so a
// sum is the same in whatever order it is made.  Logits are compared as
// 32-bit keys that ascend with them (0: never drawn).  The kept words are a
// prefix of the order (key descending, index ascending) in every setting: all
// keys above some key and the first few words at it.
//
// 1. scan: a wave reads 2048 logits, notes their largest key and lists the
//    few words whose key is at least its 24th largest lane maximum.  Together
//    the lists hold every word of the row above the largest of these bounds.
// 2. sums (only rows that need the weight of all words): the weights of each
//    2048 words added.
// 3. draw: a block per row, on the listed words in LDS wherever the kept ones
//    are among them, else on the whole row.
#include <algorithm>

#include "codes.h"
#include "mq_internal.h"

namespace mq {
namespace {

constexpr int kSeg = 2048;       // words per wave of the first two kernels
constexpr int kList = 64;        // places in a wave's list
constexpr int kRank = 24;        // lane maxima at or above a list's bound
constexpr int kDrawThreads = 512, kDrawWaves = kDrawThreads / 64;
constexpr int kBins = 2 * kDrawThreads, kBinBits = 10;
constexpr int kEntries = 8192;   // listed words that the draw takes into LDS
constexpr double kOne = 1099511627776.0;  // 2^40

struct SampleArgs {
    const void* x;
    int64_t ld;
    int32_t V, segs;
    double alpha;           // logit = alpha * (code - zp) for 16-bit codes
    int32_t zp;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    const float* u;
    int32_t* tokens;
    uint4* info;            // [rows][segs]: largest key, bound, listed words
    uint2* list;            // [rows][segs][kList]: key, index
    int64_t* sums;          // [rows][segs]
};

struct Fp32 {
    using T = float;
    static __device__ uint32_t key(float x)
    {
        uint32_t b = __float_as_uint(x);
        if (b == 0x80000000u) b = 0;           // -0 is 0
        const uint32_t k = (b >> 31) ? ~b : b | 0x80000000u;
        return !(x > -__builtin_inff()) ? 0 : k;  // NaN and -inf are never drawn
    }
    static __device__ double value(const SampleArgs&, uint32_t k)
    {
        return (double)__uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k);
    }
};
struct Code16 {
    using T = int16_t;
    static __device__ uint32_t key(int16_t q) { return (uint32_t)((int32_t)q + 32769); }
    static __device__ double value(const SampleArgs& p, uint32_t k)
    {
        return p.alpha * (double)((int32_t)k - 32769 - p.zp);
    }
};

// A row's settings.
struct Row {
    double max;      // its largest logit
    double scale;    // log2(e) / temperature
    double p, floor; // top_p (>= 1: off), least weight of the min_p rule
    int32_t k;       // 0: off
    uint32_t kmax;
};

template <class F>
__device__ inline Row row_of(const SampleArgs& a, int64_t m, uint32_t kmax)
{
    Row r;
    r.kmax = kmax;
    r.max = F::value(a, kmax);
    const double t = a.temperature ? (double)a.temperature[m] : 1.0;
    const int32_t k = a.top_k ? a.top_k[m] : 0;
    r.k = k > 0 && k < a.V ? k : 0;
    r.p = a.top_p ? (double)a.top_p[m] : 1.0;
    if (!(r.p < 1.0)) r.p = 1.0;
    const double mp = a.min_p ? (double)a.min_p[m] : 0.0;
    r.floor = mp > 0.0 ? fmin(mp, 1.0) * kOne : 0.0;
    r.scale = 1.4426950408889634 / t;
    if (!(t > 0.0)) {  // greedy: the first of the largest
        r.k = 1;
        r.scale = 1.4426950408889634;
    }
    return r;
}

template <class F>
__device__ inline int64_t weight(const SampleArgs& a, const Row& r, uint32_t k)
{
    if (k == r.kmax) return (int64_t)1 << 40;
    if (k == 0 || r.max == (double)__builtin_inff()) return 0;
    const double z = fmax((F::value(a, k) - r.max) * r.scale, -100.0);
    const double w = exp2_poly(z + 40.0) + kRintShift;
    return __double_as_longlong(w) - __double_as_longlong(kRintShift);
}

// Whether the row's draw needs the weights of all words.
__device__ inline bool needs_sums(const Row& r) { return r.k == 0; }

template <class F>
__global__ __launch_bounds__(256) void sample_scan_kernel(SampleArgs a, int64_t row0)
{
    const int lane = threadIdx.x & 63;
    const int seg = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (seg >= a.segs) return;
    const int64_t m = blockIdx.y;
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + (row0 + m) * a.ld;
    const int32_t i0 = seg * kSeg + lane;
    uint32_t k[kSeg / 64];
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) k[j] = i0 + 64 * j < a.V ? F::key(x[i0 + 64 * j]) : 0;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) top = max(top, k[j]);
    // the largest bound that kRank lanes' maxima reach
    uint32_t bound = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t c = bound | (1u << bit);
        if (__popcll(__ballot(top >= c)) >= kRank) bound = c;
    }
    bound = max(bound, 1u);  // key 0 is never listed
    int n = 0;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) n += __popcll(__ballot(k[j] >= bound));
    if (n > kList) {  // the smallest bound that leaves no more than the list holds
        uint32_t b = 0;
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = b | (1u << bit);
            int cnt = 0;
#pragma unroll
            for (int j = 0; j < kSeg / 64; ++j) cnt += __popcll(__ballot(k[j] >= c));
            if (cnt > kList) b = c;
        }
        bound = b + 1;  // b: the largest key that too many reach (b < 2^32 - 1)
    }
    const int64_t at = m * a.segs + seg;
    uint2* list = a.list + at * kList;
    int pos = 0;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int j = 0; j < kSeg / 64; ++j) {
        const uint64_t hit = __ballot(k[j] >= bound);
        if (hit) {
            if (k[j] >= bound)
                list[pos + __popcll(hit & below)] = make_uint2(k[j], (uint32_t)(i0 + 64 * j));
            pos += __popcll(hit);
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    if (lane == 0) a.info[at] = make_uint4(top, bound, (uint32_t)pos, 0);
}

// The row's largest key, from its segments (every lane of the wave).
__device__ inline uint32_t row_max(const SampleArgs& a, int64_t m)
{
    uint32_t top = 0;
    for (int i = threadIdx.x & 63; i < a.segs; i += 64) top = max(top, a.info[m * a.segs + i].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    return top;
}

template <class F>
__global__ __launch_bounds__(256) void sample_sums_kernel(SampleArgs a, int64_t row0)
{
    const int lane = threadIdx.x & 63;
    const int seg = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (seg >= a.segs) return;
    const int64_t m = blockIdx.y;
    const uint32_t kmax = row_max(a, m);
    const Row r = row_of<F>(a, row0 + m, kmax);
    if (!needs_sums(r) || kmax == 0) return;
    const typename F::T* x = static_cast<const typename F::T*>(a.x) + (row0 + m) * a.ld;
    const int32_t i0 = seg * kSeg + lane;
    // without top_p the floor alone decides what is kept
    const double least = r.p < 1.0 ? 0.0 : r.floor;
    int64_t s = 0;
#pragma unroll 4
    for (int j = 0; j < kSeg / 64; ++j) {
        const int64_t w = i0 + 64 * j < a.V ? weight<F>(a, r, F::key(x[i0 + 64 * j])) : 0;
        s += (double)w >= least ? w : 0;
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
    if (lane == 0) a.sums[m * a.segs + seg] = s;
}

// ---------------------------------------------------------------------------
// The draw.

struct DrawLds {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
    uint32_t key[kEntries];
    uint32_t idx[kEntries];
    int64_t wave64[kDrawWaves];
    int32_t wave32[kDrawWaves];
    uint32_t sel[4];
    int64_t sel64[2];
};

// Sums of one value per thread over the block: the sum of the threads before
// this one, and the total.
__device__ inline int64_t block_scan(int64_t v, int64_t* total, int64_t* lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t t = __shfl_up(s, o);
        if (lane >= o) s += t;
    }
    __syncthreads();
    if (lane == 63) lds[wave] = s;
    __syncthreads();
    int64_t before = 0, all = 0;
    for (int w = 0; w < kDrawWaves; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    *total = all;
    return before + s - v;
}

// The words that a draw looks at: the listed ones in LDS or the whole row.
template <class F>
struct Words {
    const DrawLds* lds;
    const typename F::T* x;
    int32_t n;
    bool listed;
    __device__ uint32_t key(int32_t i) const { return listed ? lds->key[i] : F::key(x[i]); }
    __device__ uint32_t index(int32_t i) const { return listed ? lds->idx[i] : (uint32_t)i; }
};

// The cut of the order where the count (MASS false) or the mass of the words
// before reaches a target: keys above `key` are kept and the first `ties` at
// it.  lo: least key that belongs to the set, lo_ties of it (the rest are
// not in the set).
struct Cut {
    uint32_t key;
    int64_t ties;
    int64_t count, mass;  // of the words above key
};

template <class F, bool MASS>
__device__ Cut find_cut(const SampleArgs& a, const Row& r, const Words<F>& ws, DrawLds& lds,
                        uint32_t lo, int64_t lo_ties, int64_t count, double mass)
{
    const int tid = threadIdx.x;
    uint32_t hi = r.kmax;
    const uint32_t set_lo = lo;
    Cut c;
    c.count = 0;
    c.mass = 0;
    for (;;) {
        const uint32_t range = hi - lo;
        const int bits = range ? 32 - __builtin_clz(range) : 0;
        const int shift = bits > kBinBits ? bits - kBinBits : 0;
        __syncthreads();
        for (int i = tid; i < kBins; i += kDrawThreads) {
            lds.count[i] = 0;
            lds.mass[i] = 0;
        }
        if (tid == 0) lds.sel[0] = 0;
        __syncthreads();
        for (int i = tid; i < ws.n; i += kDrawThreads) {
            const uint32_t k = ws.key(i);
            if (k < lo || k > hi) continue;
            const uint32_t bin = (k - lo) >> shift;
            atomicAdd(&lds.count[bin], 1u);
            atomicAdd(&lds.mass[bin], (unsigned long long)weight<F>(a, r, k));
        }
        __syncthreads();
        // from the top: thread t holds bins kBins - 1 - 2 t and the one below
        const int b0 = kBins - 1 - 2 * tid, b1 = b0 - 1;
        const int64_t n0 = lds.count[b0], n1 = lds.count[b1];
        const int64_t m0 = (int64_t)lds.mass[b0], m1 = (int64_t)lds.mass[b1];
        int64_t all;
        const int64_t nb = c.count + block_scan(n0 + n1, &all, lds.wave64);
        const int64_t mb = c.mass + block_scan(m0 + m1, &all, lds.wave64);
        // the first bin from the top that reaches the target, else the last
        // one with words
        auto reaches = [&](int64_t n, int64_t m) {
            return MASS ? (double)m >= mass : n >= count;
        };
        if (n0 && (reaches(nb + n0, mb + m0))) atomicMax(&lds.sel[0], (uint32_t)b0 + 4096);
        if (n1 && (reaches(nb + n0 + n1, mb + m0 + m1))) atomicMax(&lds.sel[0], (uint32_t)b1 + 4096);
        __syncthreads();
        if (lds.sel[0] == 0) {  // none: the lowest bin with words
            __syncthreads();
            if (tid == 0) lds.sel[1] = kBins;
            __syncthreads();
            if (n1) atomicMin(&lds.sel[1], (uint32_t)b1);
            else if (n0) atomicMin(&lds.sel[1], (uint32_t)b0);
            __syncthreads();
            if (tid == 0) lds.sel[0] = lds.sel[1] + 4096;
            __syncthreads();
        }
        const uint32_t bin = lds.sel[0] - 4096;
        if ((uint32_t)b0 == bin || (uint32_t)b1 == bin) {
            lds.sel64[0] = (uint32_t)b0 == bin ? nb : nb + n0;
            lds.sel64[1] = (uint32_t)b0 == bin ? mb : mb + m0;
        }
        __syncthreads();
        c.count = lds.sel64[0];
        c.mass = lds.sel64[1];
        lo = lo + (bin << shift);
        hi = min(hi, lo + ((1u << shift) - 1));
        if (shift == 0) {
            c.key = lo;
            int64_t ties = lds.count[bin];
            if (lo == set_lo) ties = min(ties, lo_ties);
            int64_t keep = ties;
            if (MASS) {
                const int64_t w = weight<F>(a, r, lo);
                // the fewest ties that reach the mass
                int64_t l = 1, h = ties;
                while (l < h) {
                    const int64_t mid = (l + h) >> 1;
                    if ((double)(c.mass + mid * w) >= mass) h = mid;
                    else l = mid + 1;
                }
                keep = l;
            } else {
                keep = min(ties, count - c.count);
            }
            c.ties = keep;
            return c;
        }
    }
}

// The word at which the running weight of the kept ones, in index order,
// passes u times their total; every wave walks a contiguous part.
template <class F>
__device__ int32_t draw_word(const SampleArgs& a, const Row& r, const Words<F>& ws, DrawLds& lds,
                             uint32_t cut, int64_t ties, double u)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    const int32_t part = ((ws.n + kDrawWaves - 1) / kDrawWaves + 63) & ~63;
    const int32_t i0 = min(wave * part, ws.n), i1 = min(i0 + part, ws.n);
    int32_t t = 0;
    for (int32_t i = i0; i < i1; i += 64)
        t += __popcll(__ballot(i + lane < i1 && ws.key(i + lane) == cut));
    __syncthreads();
    if (lane == 0) lds.wave32[wave] = t;
    __syncthreads();
    int64_t first = 0;  // ties before this wave's part
    for (int w = 0; w < wave; ++w) first += lds.wave32[w];

    auto kept = [&](int32_t i, int64_t& seen) -> int64_t {
        const uint32_t k = i < i1 ? ws.key(i) : 0;
        const uint64_t tie = __ballot(k == cut && i < i1);
        const int64_t rank = seen + __popcll(tie & below);
        seen += __popcll(tie);
        if (!(k > cut || (k == cut && rank < ties)) || i >= i1) return 0;
        const int64_t w = weight<F>(a, r, k);
        return (double)w >= r.floor ? w : 0;
    };
    int64_t s = 0, seen = first;
    for (int32_t i = i0; i < i1; i += 64) s += kept(i + lane, seen);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
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
        seen = first;
        int64_t run = before;
        for (int32_t i = i0; i < i1; i += 64) {
            const int64_t w = kept(i + lane, seen);
            int64_t c = w;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int64_t v = __shfl_up(c, o);
                if (lane >= o) c += v;
            }
            const uint64_t hit = __ballot(run + c > target);
            if (hit) {
                if (lane == __builtin_ctzll(hit)) lds.sel[0] = ws.index(i + lane);
                break;
            }
            run += __shfl(c, 63);
        }
    }
    __syncthreads();
    return (int32_t)lds.sel[0];
}

template <class F>
__global__ __launch_bounds__(kDrawThreads) void sample_draw_kernel(SampleArgs a, int64_t row0)
{
    __shared__ DrawLds lds;
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t m = blockIdx.x, row = row0 + m;
    const uint4* info = a.info + m * a.segs;
    const uint32_t kmax = row_max(a, m);
    if (kmax == 0) {  // nothing can be drawn
        if (tid == 0) a.tokens[row] = -1;
        return;
    }
    const Row r = row_of<F>(a, row, kmax);
    const double u0 = (double)a.u[row], u = u0 > 0.0 ? fmin(u0, 1.0) : 0.0;

    // what all lists together hold without a gap: keys from the largest bound
    uint32_t bound = 1;
    for (int i = lane; i < a.segs; i += 64) bound = max(bound, info[i].y);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) bound = max(bound, (uint32_t)__shfl_xor((int)bound, o));

    const typename F::T* x = static_cast<const typename F::T*>(a.x) + row * a.ld;
    Words<F> ws{&lds, x, a.V, false};

    // listed words into LDS, in index order; a thread per segment and turn
    int64_t n = 0;
    for (int s0 = 0; s0 < a.segs; s0 += kDrawThreads) {
        const int s = s0 + tid;
        const uint2* list = a.list + (m * a.segs + s) * kList;
        const int cnt = s < a.segs ? (int)info[s].z : 0;
        int mine = 0;
        for (int i = 0; i < cnt; ++i) mine += list[i].x >= bound;
        int64_t all;
        int64_t at = n + block_scan(mine, &all, lds.wave64);
        for (int i = 0; i < cnt; ++i)
            if (list[i].x >= bound) {
                if (at < kEntries) {
                    lds.key[at] = list[i].x;
                    lds.idx[at] = list[i].y;
                }
                ++at;
            }
        n += all;
    }
    __syncthreads();
    const bool have_list = n > 0 && n <= kEntries;

    if (needs_sums(r) && !(r.p < 1.0)) {
        // no cut: the segment, then the word in it
        int64_t s = 0, all = 0, base = 0, total = 0;
        for (int i = tid; i < a.segs; i += kDrawThreads) s += a.sums[m * a.segs + i];
        block_scan(s, &total, lds.wave64);
        const int64_t target = min((int64_t)(u * (double)total), total - 1);
        if (tid == 0) lds.sel[0] = 0;
        __syncthreads();
        for (int s0 = 0; s0 < a.segs; s0 += kDrawThreads) {
            const int i = s0 + tid;
            const int64_t v = i < a.segs ? a.sums[m * a.segs + i] : 0;
            const int64_t before = base + block_scan(v, &all, lds.wave64);
            if (target >= before && target < before + v) {
                lds.sel[0] = (uint32_t)i;
                lds.sel64[0] = before;
            }
            base += all;
        }
        __syncthreads();
        if (tid >= 64) return;
        const int32_t i0 = (int32_t)lds.sel[0] * kSeg, i1 = min(i0 + kSeg, a.V);
        int64_t run = lds.sel64[0];
        for (int32_t i = i0; i < i1; i += 64) {
            int64_t c = i + lane < i1 ? weight<F>(a, r, F::key(x[i + lane])) : 0;
            if (!((double)c >= r.floor)) c = 0;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int64_t v = __shfl_up(c, o);
                if (lane >= o) c += v;
            }
            const uint64_t hit = __ballot(run + c > target);
            if (hit) {
                if (lane == __builtin_ctzll(hit)) a.tokens[row] = i + lane;
                return;
            }
            run += __shfl(c, 63);
        }
        return;
    }

    uint32_t cut = 1;
    int64_t ties = INT64_MAX, total;
    if (r.k > 0) {
        ws.listed = have_list && n >= r.k;
        ws.n = ws.listed ? (int32_t)n : a.V;
        const Cut c = find_cut<F, false>(a, r, ws, lds, ws.listed ? bound : 1, INT64_MAX, r.k, 0.0);
        cut = c.key;
        ties = c.ties;
        total = c.mass + c.ties * weight<F>(a, r, c.key);
    } else {
        int64_t s = 0;
        for (int i = tid; i < a.segs; i += kDrawThreads) s += a.sums[m * a.segs + i];
        block_scan(s, &total, lds.wave64);
    }
    if (r.p < 1.0) {
        const double mass = r.p * (double)total;
        if (r.k == 0 && have_list) {
            // listed words hold the mass?
            int64_t s = 0, all;
            for (int i = tid; i < n; i += kDrawThreads) s += weight<F>(a, r, lds.key[i]);
            block_scan(s, &all, lds.wave64);
            ws.listed = (double)all >= mass;
            ws.n = ws.listed ? (int32_t)n : a.V;
        }
        const uint32_t lo = r.k > 0 ? cut : ws.listed ? bound : 1;
        const Cut c = find_cut<F, true>(a, r, ws, lds, lo, ties, 0, mass);
        cut = c.key;
        ties = c.ties;
    }
    const int32_t tok = draw_word<F>(a, r, ws, lds, cut, ties, u);
    if (tid == 0) a.tokens[row] = tok;
}

int32_t segments(int64_t V) { return (int32_t)((V + kSeg - 1) / kSeg); }

// Bytes per row of the three workspace parts.
int64_t row_bytes(int64_t V) { return (int64_t)segments(V) * (16 + 8 * kList + 8); }

template <class F>
hipError_t launch(SampleArgs a, int64_t M, char* ws, int64_t ws_bytes, hipStream_t s)
{
    const int64_t rows = std::min<int64_t>(ws_bytes / row_bytes(a.V), 65535);
    for (int64_t m0 = 0; m0 < M; m0 += rows) {
        const int64_t n = std::min(rows, M - m0);
        a.info = reinterpret_cast<uint4*>(ws);
        a.list = reinterpret_cast<uint2*>(ws + n * a.segs * 16);
        a.sums = reinterpret_cast<int64_t*>(ws + n * a.segs * (16 + 8 * kList));
        const dim3 g((unsigned)((a.segs + 3) / 4), (unsigned)n);
        sample_scan_kernel<F><<<g, 256, 0, s>>>(a, m0);
        sample_sums_kernel<F><<<g, 256, 0, s>>>(a, m0);
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
                         int32_t zp, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, const float* u, int32_t* tokens,
                         void* ws, int64_t ws_bytes, hipStream_t s)
{
    SampleArgs a;
    a.x = x;
    a.ld = ld;
    a.V = (int32_t)V;
    a.segs = segments(V);
    a.alpha = alpha;
    a.zp = zp;
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
