// Attention of new tokens over the paged key/value cache, scores and weights
// in registers throughout.
//
// A wave holds 16 rows (a row: one token's query head; the H / G heads that
// share a cache head lie next to each other) and walks over blocks of 128 key
// positions.  Products run on the int8 matrix instructions, 16-bit operands
// split into two byte planes.  Scores come out transposed,
//   C[key][row] = K[key][d] * Q[row][d],
// a lane holding one row (lane & 15) and, the 16 keys of a tile being taken
// in the order 16 (r >> 2) + 4 j + (r & 3), 16 consecutive keys per 64: the
// layout that the second product takes as its operand,
//   O[d][row] = V^T[d][key] * W[key][row],
// so the weights go from one product to the other without leaving the lane,
// and a row's maximum, weight sum and factors live where its outputs do.
//
// Scores of a block are exact, so its weights are integers relative to its own
// maximum and its sums exact; only the factors between blocks and the sums of
// these products are fp64.  Fewer bits anywhere: none but the weights' 15.
//
// Vector arithmetic bounds it where many rows share keys (13 instructions and
// two reads across lanes per weight, of 4.4 cycles each; the products of the
// same block take 1000 of its 8500 cycles at D = 128), the way to memory
// (page list, keys, values, each waiting for the one before) where few do.
// Rows of several waves share the keys: these come once into LDS, by copies
// that need no registers, and a CU's two work-groups overlap.  Few rows are one
// wave's, so the keys are split instead, among four waves and among work-groups.
// us, kernel (and join) traced in a row: one token over 1531 keys, 32 heads of
// 64 on 4, 7.5 (3.3); 64 tokens over up to 4096, 67 MB, 23.7 (4.0); 2 over up
// to 120000, 8 heads of 256 on 1, 61 MB, 26.2 (4.7); 24 windows of 1000, 46 MB,
// 20.9; a prompt of 1024, 29.0; 500 tokens over 16000, 32 heads of 128 on 8, 282
// (12.8): 0.92 POP/s of int8 products.  A call in a row without the tracer:
// 12.3, 25.6, 31.5, 21.5, 25.0, 287.
#include <algorithm>
#include <cmath>

#include "codes.h"
#include "kvcache.h"
#include "mq_internal.h"
#include "requant.h"

#define MQ_LDS __attribute__((address_space(3)))
#define MQ_GLOBAL __attribute__((address_space(1)))

namespace mq {
namespace {

constexpr int kBlk = MQ_ATTN_BLOCK;
constexpr int kRows = 16;             // rows per wave
constexpr int kWaves = 4;             // waves per work-group
constexpr int kTile = kRows * kWaves; // rows per work-group where the waves share keys
constexpr int kMaxSplits = 256;
constexpr int32_t kNone = INT32_MIN;  // no key seen (|c| <= 65535 * 128 * 256 < 2^31)

struct AttnArgs {
    KvArgs kv;
    const int16_t* q;
    void* y;
    int64_t ldq, ldy, T;
    int32_t H, grp;       // grp = H / G
    int32_t q_zp, v_zp, out_zp, out_bits;
    double tau;           // log2(e) * q_scale * k_scale * logit_scale
    double v_scale, out_scale;
    uint32_t d_cut;       // logit distances from here on weigh nothing
    int32_t window, sinks; // window 0: none
    int32_t page_bytes;    // of a page's keys, and of its values (at most 2^28)
    int32_t vec_q, vec_y; // query rows in 16-byte chunks, output rows in fours of codes
    int32_t splits;
    double* mz;           // [T * H][splits][2]: maximum and weight sum of a part
    double* sums;         // [T * H][splits][D]
};

// factor between two block maxima, 2^(-tau (hi - lo)), hi >= lo
__device__ inline double factor(const AttnArgs& p, int32_t hi, int32_t lo)
{
    return exp2_poly(fmax(-p.tau * ((double)hi - (double)lo), -1000.0));
}

__device__ inline v4i mfma(v4i a, v4i b, v4i c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// The larger of a value's copies in the four lanes of one row.
__device__ inline int32_t row_max(int32_t m)
{
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)m, (uint32_t)m, false, false);
    m = max((int32_t)a[0], (int32_t)a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)m, (uint32_t)m, false, false);
    return max((int32_t)b[0], (int32_t)b[1]);
}

// rint(MQ_ATTN_ONE 2^(-tau d)) + 128 for 0 <= tau d < 1000: tau d to the next
// 1/64, 2^(j/64) from the table that the wave's lanes hold (lane j), exp2_rest
// and the last product added to 1.5 * 2^52 + 128, whose low word is then the
// rounded weight and 128.  The high words of the table lack j << 14, which
// k << 14 (k = 64 n + j) adds again with the exponent n.  11 vector instructions
// and two reads across lanes; the polynomial over all of [-1/2, 1/2] (degree
// 10) took 18.
constexpr int32_t kBias = 128;
struct WeightTable {
    int lo, hi;  // MQ_ATTN_ONE * 2^(lane/64)
    __device__ void init()
    {
        const int lane = threadIdx.x & 63;
        const double e = (double)MQ_ATTN_ONE * exp2_poly((double)lane / 64.0);
        lo = (int)(uint32_t)__double_as_longlong(e);
        hi = (int)(__double_as_longlong(e) >> 32) - (lane << 14);
    }
    // A weight on its way: the table's reads take a while.
    struct Part {
        double f;
        int k, lo, hi;
    };
    __device__ Part begin(double tau, uint32_t d) const
    {
        Part w;
        const double x = (double)d;
        const double t = __builtin_fma(-tau, x, kTableShift);
        w.f = __builtin_fma(-tau, x, -(t - kTableShift));
        w.k = rint_low(t);
        w.lo = __builtin_amdgcn_ds_bpermute(w.k << 2, lo);
        w.hi = __builtin_amdgcn_ds_bpermute(w.k << 2, hi);
        // computed here, not where it is used
        asm volatile("" : "+v"(w.f), "+v"(w.k));
        return w;
    }
    __device__ static int32_t end(const Part& w)
    {
        const double e =
            __longlong_as_double(((int64_t)(w.hi + (w.k << 14)) << 32) | (uint32_t)w.lo);
        return rint_low(__builtin_fma(exp2_rest(w.f), e, kRintShift + kBias));
    }
};

// Four weights (each with kBias) as two planes of signed bytes, w = 256 hi +
// lo: the bias makes byte 1 the one, byte 0 less 128 the other.
__device__ inline void pack_weights4(const int32_t* w, int& hi, int& lo)
{
    const uint32_t p = __builtin_amdgcn_perm((uint32_t)w[1], (uint32_t)w[0], 0x05010400u);
    const uint32_t q = __builtin_amdgcn_perm((uint32_t)w[3], (uint32_t)w[2], 0x05010400u);
    lo = (int)(__builtin_amdgcn_perm(q, p, 0x05040100u) ^ 0x80808080u);
    hi = (int)__builtin_amdgcn_perm(q, p, 0x07060302u);
}

// The state of a wave's 16 rows.
template <int KS, int ND>
struct Rows {
    v4i qh[KS], ql[KS];     // byte planes of the queries
    int32_t cz;
    double acc[ND][4];      // output channels 16 dt + 4 (lane >> 4) + i of row lane & 15
    double z;
    int32_t m;
    __device__ void clear()
    {
        m = kNone;
        z = 0.0;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[dt][i] = 0.0;
    }
};

template <int KS>
__device__ inline void load_queries(const AttnArgs& p, int64_t t, int32_t head, bool have,
                                    v4i (&qh)[KS], v4i (&ql)[KS], int32_t& cz)
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int16_t* x = p.q + t * p.ldq + (int64_t)head * p.kv.D;
    bool fits = true;
    v4i raw[KS][2];
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = 64 * s + 16 * g;
        int32_t c[16];
        if (have && d < p.kv.D) {
            if (p.vec_q) {
                raw[s][0] = *reinterpret_cast<const v4i*>(x + d);
                raw[s][1] = *reinterpret_cast<const v4i*>(x + d + 8);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t a = (uint16_t)x[d + 2 * i], b = (uint16_t)x[d + 2 * i + 1];
                    raw[s][i >> 2][i & 3] = (int)(a | (b << 16));
                }
            }
            unpack8(raw[s][0], c);
            unpack8(raw[s][1], c + 8);
        } else {
            // channels past the head and rows past the tile: q = q_zp
            const uint32_t z = (uint16_t)p.q_zp;
#pragma unroll
            for (int i = 0; i < 8; ++i) raw[s][i >> 2][i & 3] = (int)(z | (z << 16));
#pragma unroll
            for (int i = 0; i < 16; ++i) c[i] = p.q_zp;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t h = 0, l = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int32_t v = c[4 * i + j] - p.q_zp, hi = (v + 128) >> 8;
                fits = fits && hi >= -128 && hi <= 127;
                h |= (uint32_t)(uint8_t)hi << (8 * j);
                l |= (uint32_t)(uint8_t)v << (8 * j);
            }
            qh[s][i] = (int)h;
            ql[s][i] = (int)l;
        }
    }
    // q - q_zp in two signed bytes where every code of the tile allows it;
    // else the code's own bytes, q = 256 h + l + 128, and 128 - q_zp times
    // the key's sum
    cz = 0;
    if (__ballot(!fits) != 0) {
        cz = 128 - p.q_zp;
#pragma unroll
        for (int s = 0; s < KS; ++s) split_a16(raw[s][0], raw[s][1], qh[s], ql[s]);
    }
}

// What one row sees: positions (lo, hi], and below the sinks.
struct Sees {
    int32_t lo, hi;
};

// Where a lane reads a block's keys and values of half h: the key row
// 16 (r >> 2) + (r & 3) of tile 0 (tile j: 4 j rows on) from channel 16 g on,
// and 16 values of channel r from key 16 g on.  `base` is the address in page
// 0 and slot 0 of the block, `group` the lane whose page it is.  Groups
// without a place get page 0's (they are masked).
struct Spot {
    const MQ_GLOBAL int8_t* base;
    int32_t group;
    __device__ static Spot key(const AttnArgs& p, int32_t g0, int h)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
        const int32_t slot = (64 * h + 16 * (r >> 2)) & ((1 << p.kv.shift) - 1);
        return Spot{(const MQ_GLOBAL int8_t*)p.kv.k +
                        ((((int64_t)g0 << p.kv.shift) + slot + (r & 3)) * p.kv.D + 16 * g),
                    4 * h + (r >> 2)};
    }
    __device__ static Spot value(const AttnArgs& p, int32_t g0, int h)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
        const int32_t slot = (64 * h + 16 * g) & ((1 << p.kv.shift) - 1);
        return Spot{(const MQ_GLOBAL int8_t*)p.kv.v +
                        ((((int64_t)g0 * p.kv.D + r) << p.kv.shift) + slot),
                    4 * h + g};
    }
    // in the block's page; slot: bytes from the page's start to the block (a
    // page of more than 128 slots)
    __device__ const MQ_GLOBAL int8_t* at(const AttnArgs& p, int32_t pages, int32_t slot) const
    {
        const uint32_t pg = (uint32_t)max(__shfl(pages, group), 0);
        return base + ((uint64_t)pg * (uint32_t)p.page_bytes + (uint32_t)slot);
    }
};
__device__ inline int32_t block_slot(const AttnArgs& p, int32_t blk)
{
    return (blk * kBlk) & ((1 << p.kv.shift) - 1);
}

// Channels are taken in steps of 64 (KS of them) by the scores and in tiles of
// 16 (ND, an even number) by the outputs; what is past the head dimension
// there reads the head's first channels.  For the scores the query planes are
// neutral there, the outputs of such a tile are dropped.

// Offset of the lane's chunk of a key row in 64-channel step s from that in
// step 0.
__device__ inline int32_t key_chunk(const AttnArgs& p, int s)
{
    const int32_t c = 16 * ((threadIdx.x & 63) >> 4);
    return 64 * s + c < p.kv.D ? 64 * s : -c;
}
// Offset of output tile dt's values from tile 0's.
__device__ inline int32_t value_tile(const AttnArgs& p, int dt)
{
    return 16 * dt < p.kv.D ? (16 * dt) << p.kv.shift : 0;
}

// Fragments of a block straight from the cache.
template <int KS>
struct FromCache {
    // One wave per SIMD: registers for reads well ahead.  Four key tiles at once
    // and eight value tiles from the weights on took 2 sequences of 120000 keys
    // from 34.1 us to 31.6 (all sixteen: 33.6); with three waves per SIMD there
    // are no registers for it (spills).
    static constexpr bool kAhead = KS >= 3;
    const MQ_GLOBAL int8_t* k[2];
    const MQ_GLOBAL int8_t* v[2];
    const AttnArgs& p;
    __device__ FromCache(const AttnArgs& a, int32_t g0, int32_t blk, int32_t pages) : p(a)
    {
        const int32_t slot = block_slot(p, blk);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            k[h] = Spot::key(p, g0, h).at(p, pages, slot * p.kv.D);
            v[h] = Spot::value(p, g0, h).at(p, pages, slot);
        }
    }
    // The same fragments, to be read anew (their registers are not kept).
    __device__ FromCache again() const
    {
        FromCache o = *this;
        asm volatile("" : "+v"(o.k[0]), "+v"(o.k[1]));
        return o;
    }
    __device__ v4i key(int h, int j, int s) const
    {
        return *reinterpret_cast<const MQ_GLOBAL v4i*>(k[h] + (4 * j * p.kv.D + key_chunk(p, s)));
    }
    __device__ v4i value(int h, int dt) const
    {
        return *reinterpret_cast<const MQ_GLOBAL v4i*>(v[h] + value_tile(p, dt));
    }
};

// Fragments staged in LDS in the order of the lanes: 1 KB each, keys (h, j, s)
// then values (h, dt).
template <int KS, int ND>
struct FromLds {
    static constexpr bool kAhead = false;
    const MQ_LDS int8_t* at;  // of this lane
    __device__ FromLds again() const
    {
        FromLds o = *this;
        asm volatile("" : "+v"(o.at));
        return o;
    }
    __device__ v4i key(int h, int j, int s) const
    {
        return *reinterpret_cast<const MQ_LDS v4i*>(at + ((4 * h + j) * KS + s) * 1024);
    }
    __device__ v4i value(int h, int dt) const
    {
        return *reinterpret_cast<const MQ_LDS v4i*>(at + (8 * KS + ND * h + dt) * 1024);
    }
};
template <int KS, int ND>
constexpr int kStage = (8 * KS + 2 * ND) * 1024;

// The wave's own copies into LDS have landed (they count as vector memory).
__device__ inline void wait_staged()
{
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // vmcnt(0), the others left alone
}

// A wave's share of a block into a stage: two of the eight key tiles and half
// of one half's values.
template <int KS, int ND>
struct Stager {
    Spot key, value;
    int32_t last;  // key_chunk of the last step (the others are 64 s)
    __device__ Stager(const AttnArgs& p, int32_t g0, int wave)
    {
        key = Spot::key(p, g0, wave >> 1);
        key.base += (8 * (wave & 1)) * p.kv.D;
        value = Spot::value(p, g0, wave & 1);
        last = key_chunk(p, KS - 1);
    }
    __device__ void operator()(const AttnArgs& p, int32_t blk, int32_t pages, int wave,
                               MQ_LDS int8_t* stage) const
    {
        const int32_t slot = block_slot(p, blk);
        const MQ_GLOBAL int8_t* k = key.at(p, pages, slot * p.kv.D);
        const MQ_GLOBAL int8_t* v = value.at(p, pages, slot);
        MQ_LDS int8_t* ks = stage + (2 * wave * KS) * 1024;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                __builtin_amdgcn_global_load_lds(
                    (const MQ_GLOBAL void*)(k + (4 * j * p.kv.D + (s < KS - 1 ? 64 * s : last))),
                    (MQ_LDS void*)(ks + (j * KS + s) * 1024), 16, 0, 0);
        MQ_LDS int8_t* vs = stage + (8 * KS + ND * (wave & 1) + (wave >> 1)) * 1024;
#pragma unroll
        for (int i = 0; i < ND / 2; ++i)
            __builtin_amdgcn_global_load_lds(
                (const MQ_GLOBAL void*)(v + value_tile(p, 2 * i + (wave >> 1))),
                (MQ_LDS void*)(vs + 2 * i * 1024), 16, 0, 0);
    }
};

// One block of 128 positions for the wave's rows.  pages: of its groups;
// full: every row sees all of its positions that have a place.
template <int KS, int ND, class Source>
__device__ inline void attend_block(const AttnArgs& p, const WeightTable& table, Rows<KS, ND>& st,
                                    const Source& src, int32_t pages, int32_t blk,
                                    const Sees& sees, bool full)
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const v4i zero = {0, 0, 0, 0};
    const v4i ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};

    // scores of keys 64 h + 16 g + 4 j + i; J of the eight tiles at once, the
    // next ones' fragments read before these are multiplied
    v4i c[2][4];
    {
        constexpr int J = Source::kAhead ? 4 : 2, N = 8 / J;
        v4i kf[2][J][KS];
#pragma unroll
        for (int n = 0; n <= N; ++n) {
            if (n < N) {
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int s = 0; s < KS; ++s)
                        kf[n & 1][j][s] = src.key((n * J + j) >> 2, (n * J + j) & 3, s);
                __builtin_amdgcn_sched_barrier(0);
            }
            if (n == 0) continue;
            v4i hi[J], lo[J];
            const auto& k = kf[(n - 1) & 1];
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    hi[j] = mfma(k[j][s], st.qh[s], s ? hi[j] : zero);
                    lo[j] = mfma(k[j][s], st.ql[s], s ? lo[j] : zero);
                }
#pragma unroll
            for (int j = 0; j < J; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    c[((n - 1) * J + j) >> 2][((n - 1) * J + j) & 3][i] = (hi[j][i] << 8) + lo[j][i];
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (st.cz != 0) {
        const Source again = src.again();
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v4i k1 = zero;
#pragma unroll
                for (int s = 0; s < KS; ++s) k1 = mfma(again.key(h, j, s), ones, k1);
#pragma unroll
                for (int i = 0; i < 4; ++i) c[h][j][i] += __mul24(k1[i], st.cz);
            }
    }

    // the values' fragments: some from here on, or the first of them before the
    // last of the weights
    constexpr int E = 2, NV = ND / E;  // output tiles at once
    constexpr int kGroups = Source::kAhead ? 4 : 2;
    v4i v[kGroups][E][2];
    auto read_values = [&](int n) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            v[n % kGroups][e][0] = src.value(0, n * E + e);
            v[n % kGroups][e][1] = src.value(1, n * E + e);
        }
    };
    if constexpr (Source::kAhead) {
#pragma unroll
        for (int n = 0; n < kGroups; ++n) read_values(n);
        __builtin_amdgcn_sched_barrier(0);
    }

    // the largest that the row sees, without what has no place
    const uint32_t placed = (uint32_t)__ballot(pages >= 0) & 0xff;
    const bool mask = !full || placed != 0xff;
    uint32_t seen = 0xffffffffu;  // bit 16 h + 4 j + i
    if (mask) {
        // of the 16 keys of a half from `first` on those below n, as bits
        auto below = [](int32_t n, int32_t first) {
            return (1u << max(min(n - first, 16), 0)) - 1;  // n >= 0
        };
        seen = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t first = blk * kBlk + 64 * h + 16 * g;
            uint32_t bits = below(sees.hi + 1, first);
            bits &= ~below(sees.lo + 1, first) | below(p.sinks, first);
            if (!((placed >> (4 * h + g)) & 1)) bits = 0;
            seen |= bits << (16 * h);
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int keep = __builtin_amdgcn_sbfe((int)seen, i, 1);  // all ones or 0
            const int x = c[i >> 4][(i >> 2) & 3][i & 3];
            c[i >> 4][(i >> 2) & 3][i & 3] = (x & keep) | (kNone & ~keep);
        }
    }
    int32_t m = kNone;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, c[i >> 4][(i >> 2) & 3][i & 3]);
    m = row_max(m);

    const int32_t m_new = max(st.m, m);
    const double f = factor(p, m_new, m);

    // weights
    v4i wh[2], wl[2];
    // so many weights begin before the last so many end (registers for three
    // waves per SIMD where the state is small)
    constexpr int A = KS == 1 ? 2 : 4, N = 32 / A;
    WeightTable::Part part[2][A];
    int32_t w[4];
#pragma unroll
    for (int n = 0; n <= N; ++n) {
        if (n < N) {
#pragma unroll
            for (int i = 0; i < A; ++i) {
                const int x = A * n + i;
                part[n & 1][i] = table.begin(
                    p.tau, min((uint32_t)m - (uint32_t)c[x >> 4][(x >> 2) & 3][x & 3], p.d_cut));
            }
        }
        if (!Source::kAhead && n == N) read_values(0);
        __builtin_amdgcn_sched_barrier(0);
        if (n == 0) continue;
#pragma unroll
        for (int i = 0; i < A; ++i)
            w[(A * (n - 1) + i) & 3] = WeightTable::end(part[(n - 1) & 1][i]);
        if (A * n % 4 == 0) {
            const int x = A * n / 4 - 1;
            int hi4, lo4;
            pack_weights4(w, hi4, lo4);
            asm volatile("" : "+v"(hi4), "+v"(lo4));
            wh[x >> 2][x & 3] = hi4;
            wl[x >> 2][x & 3] = lo4;
        } else {
            asm volatile("" : "+v"(w[0]), "+v"(w[1]));
        }
        __builtin_amdgcn_sched_barrier(0);
    }

    if (mask) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // four bits to four bytes
                const uint32_t bits = (seen >> (16 * h + 4 * j)) & 15;
                const int keep = (int)(((bits * 0x00204081u) & 0x01010101u) * 255u);
                wh[h][j] &= keep;
                wl[h][j] &= keep;
            }
    }

    // the block joins the rows' state
    if (__ballot(m > st.m) != 0) {
        const double rs = factor(p, m_new, st.m);
        st.z *= rs;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.acc[dt][i] *= rs;
        st.m = m_new;
    }
    {
        const v4i hi = mfma(ones, wh[1], mfma(ones, wh[0], zero));
        const v4i lo = mfma(ones, wl[1], mfma(ones, wl[0], zero));
        st.z = __builtin_fma(f, (double)((hi[0] << 8) + lo[0]), st.z);
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
        if (!Source::kAhead && n + 1 < NV) {
            read_values(n + 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        const auto& x = v[n % kGroups];
        v4i hi[E], lo[E];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                hi[e] = mfma(x[e][h], wh[h], h ? hi[e] : zero);
                lo[e] = mfma(x[e][h], wl[h], h ? lo[e] : zero);
            }
        if (Source::kAhead && n + kGroups < NV) read_values(n + kGroups);
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                st.acc[n * E + e][i] = __builtin_fma(f, (double)((hi[e][i] << 8) + lo[e][i]),
                                                     st.acc[n * E + e][i]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The code of a row's channel, y / out_scale = (sum f S - v_zp z) unit with
// unit = v_scale / (z out_scale): one division per row, three roundings to
// 2^-53.  With a division by z and one by out_scale per channel a prompt of
// 1024 took 26.7 us instead of 25.0, one token of 8 heads of 256 over 30 keys
// 14.7 instead of 13.2.
__device__ inline double out_unit(const AttnArgs& p, double z)
{
    return z > 0.0 ? p.v_scale / (z * p.out_scale) : 0.0;
}
__device__ inline int32_t out_code(const AttnArgs& p, double s, double z, double unit)
{
    const double t = limit_quotient(__builtin_fma(-(double)p.v_zp, z, s) * unit);
    const int32_t q = rint_low(t + kRintShift) + p.out_zp;
    return p.out_bits == 8 ? clamp_code<8>(q) : clamp_code<16>(q);
}

__device__ inline void store_out(const AttnArgs& p, int64_t t, int32_t head, int32_t d, int32_t q)
{
    const int64_t at = t * p.ldy + (int64_t)head * p.kv.D + d;
    if (p.out_bits == 8) static_cast<int8_t*>(p.y)[at] = (int8_t)q;
    else static_cast<int16_t*>(p.y)[at] = (int16_t)q;
}

// A tile of rows of one sequence and the blocks that its rows see.  Positions
// are below 2^31 and above -2^26 (lengths are int32).
struct Tile {
    int32_t b;
    int32_t s0, pos0;         // the sequence's first token row and its position
    uint32_t row0, rows;      // first row (token, head of the group), the sequence's rows
    int32_t n, skip0, skip1;  // blocks to walk: n, without those in [skip0, skip1)
    int32_t hi_min, hi_max;   // positions of the first and last token
    int32_t last;             // of the page list's entries, the last one that a row sees
    __device__ int32_t block(int32_t i) const { return i < skip0 ? i : i + (skip1 - skip0); }
    // Every row sees all positions of the block.
    __device__ bool full(const AttnArgs& p, int32_t blk) const
    {
        return blk * kBlk + (kBlk - 1) <= hi_min &&
               (p.window == 0 || blk * kBlk > hi_max - p.window);
    }
};

// The page list's entries for a block's eight 16-key groups, in the lanes' low
// three bits, as they are (looked at when the block's turn comes, so that the
// load can be under way until then).  Entries past the tile's last are not read.
__device__ inline int32_t page_entry(const AttnArgs& p, int32_t blk)
{
    return (blk * kBlk + 16 * (int32_t)(threadIdx.x & 7)) >> p.kv.shift;
}
__device__ inline int32_t load_pages(const AttnArgs& p, const Tile& t, int32_t blk)
{
    return p.kv.table[(int64_t)t.b * p.kv.ld + min(page_entry(p, blk), t.last)];
}
// Those that are a place in the cache, else -1.
__device__ inline int32_t valid_pages(const AttnArgs& p, const Tile& t, int32_t blk, int32_t pages)
{
    return page_entry(p, blk) <= t.last && pages >= 0 && pages < (int32_t)p.kv.pages ? pages : -1;
}

// The tile's index counts from floor(starts[b] grp / R) + b for sequence b: an
// upper bound of the tiles before it that needs no scan.
template <int R>
__device__ inline bool find_tile(const AttnArgs& p, int64_t index, Tile& t)
{
    const int32_t* starts = p.kv.starts;
    const int32_t grp = p.grp;
    t.b = find_seq(p.kv.B, index, [=](int32_t i) { return (int64_t)starts[i] * grp / R + i; });
    const int32_t s0 = starts[t.b], s1 = starts[t.b + 1], len = max(p.kv.lens[t.b], 0);
    if (s0 < 0 || s1 > (int32_t)p.T || s0 >= s1) return false;
    const int64_t row0 = (index - ((int64_t)s0 * grp / R + t.b)) * R;
    t.s0 = s0;
    t.rows = (uint32_t)(s1 - s0) * (uint32_t)grp;  // below 2^32 (T H D is below 2^36)
    if (row0 < 0 || row0 >= (int64_t)t.rows) return false;
    t.row0 = (uint32_t)row0;
    t.pos0 = len - (s1 - s0);
    t.hi_max = t.pos0 + (int32_t)((min(t.row0 + (R - 1), t.rows - 1)) / (uint32_t)grp);
    t.hi_min = t.pos0 + (int32_t)(t.row0 / (uint32_t)grp);
    // blocks with places, up to the last row's
    const int64_t list = ((p.kv.ld << p.kv.shift) + kBlk - 1) / kBlk;
    const int32_t end = t.hi_max < 0 ? 0 : (int32_t)min((int64_t)(t.hi_max / kBlk + 1), list);
    t.last = (int32_t)min((int64_t)(t.hi_max >> p.kv.shift), p.kv.ld - 1);
    t.skip0 = t.skip1 = 0;
    if (p.window > 0) {
        t.skip1 = t.hi_min >= p.window ? min((t.hi_min - p.window + 1) / kBlk, end) : 0;
        t.skip0 = min((int32_t)(((int64_t)p.sinks + kBlk - 1) / kBlk), t.skip1);
    }
    t.n = end - (t.skip1 - t.skip0);
    return true;
}

// Row lane & 15 of the 16 from `first` on: token row, query head, what it sees.
struct RowAt {
    bool have;
    int64_t t;
    int32_t head;
    Sees sees;
    __device__ RowAt(const AttnArgs& p, const Tile& tile, uint32_t first, int32_t g0)
    {
        const uint32_t x = first + (threadIdx.x & 15);  // no overflow: rows below 2^32 - 64
        have = x < tile.rows;
        const uint32_t row = have ? x : tile.rows - 1, tok = row / (uint32_t)p.grp;
        t = (int64_t)tile.s0 + tok;
        head = g0 * p.grp + (int32_t)(row - tok * (uint32_t)p.grp);
        sees.hi = max(tile.pos0 + (int32_t)tok, -1);
        sees.lo = p.window > 0 && sees.hi >= p.window ? sees.hi - p.window : -1;
    }
};

// Four waves share 16 rows and take every fourth block of [i0, i1); their
// states are joined through LDS, J output tiles at a time.
template <int J>
constexpr int kJoinDoubles = J * kWaves * 4 * 64 + kWaves * kRows * 3 / 2;
template <int KS, int ND, int J>
__device__ inline void split_rows(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, int split, double* lds)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowAt row(p, tile, tile.row0, g0);
    Rows<KS, ND> st;
    st.clear();
    int32_t i = i0 + wave;
    if (i < i1) {
        WeightTable table;
        table.init();
        int32_t pages = load_pages(p, tile, tile.block(i));
        load_queries<KS>(p, row.t, row.head, row.have, st.qh, st.ql, st.cz);
        for (; i < i1; i += kWaves) {
            const int32_t blk = tile.block(i);
            pages = valid_pages(p, tile, blk, pages);
            const FromCache<KS> src(p, g0, blk, pages);
            const int32_t next = load_pages(p, tile, tile.block(min(i + kWaves, i1 - 1)));
            attend_block<KS, ND>(p, table, st, src, pages, blk, row.sees, tile.full(p, blk));
            pages = next;
        }
    }

    double* lz = lds + J * kWaves * 4 * 64;                              // [wave][row]
    int32_t* lm = reinterpret_cast<int32_t*>(lz + kWaves * kRows);       // [wave][row]
    if (g == 0) {
        lm[wave * kRows + r] = st.m;
        lz[wave * kRows + r] = st.z;
    }
    __syncthreads();
    int32_t m = kNone;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = max(m, lm[w * kRows + r]);
    double z = 0.0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
        z = __builtin_fma(factor(p, m, lm[w * kRows + r]), lz[w * kRows + r], z);
    const double f = factor(p, m, st.m);
    const int64_t at = (row.t * p.H + row.head) * p.splits + split;
    if (p.splits > 1 && row.have && wave == 0 && g == 0) {
        p.mz[2 * at] = (double)m;
        p.mz[2 * at + 1] = z;
    }
    const double unit = out_unit(p, z);
#pragma unroll
    for (int d0 = 0; d0 < ND; d0 += J) {
        if (16 * d0 >= p.kv.D) break;
        if (d0) __syncthreads();
#pragma unroll
        for (int e = 0; e < J && d0 + e < ND; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                lds[((e * kWaves + wave) * 4 + i) * 64 + lane] = f * st.acc[d0 + e][i];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < J && d0 + e < ND; ++e) {
            double s = 0.0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += lds[((e * kWaves + w) * 4 + wave) * 64 + lane];
            const int32_t d = 16 * (d0 + e) + 4 * g + wave;
            if (row.have && d < p.kv.D) {
                if (p.splits > 1) p.sums[at * p.kv.D + d] = s;
                else store_out(p, row.t, row.head, d, out_code(p, s, z, unit));
            }
        }
    }
}

// Every wave has 16 rows of its own; all walk over blocks [i0, i1), staged in
// LDS by the four together, the next block on its way during this one.
template <int KS, int ND>
__device__ inline void share_keys(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, int split, MQ_LDS int8_t* lds)
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowAt row(p, tile, tile.row0 + kRows * wave, g0);
    Rows<KS, ND> st;
    st.clear();
    if (i0 < i1) {
        WeightTable table;
        table.init();
        int32_t pages = valid_pages(p, tile, tile.block(i0), load_pages(p, tile, tile.block(i0)));
        const Stager<KS, ND> stage(p, g0, wave);
        stage(p, tile.block(i0), pages, wave, lds);
        int32_t next = load_pages(p, tile, tile.block(min(i0 + 1, i1 - 1)));
        load_queries<KS>(p, row.t, row.head, row.have, st.qh, st.ql, st.cz);
        wait_staged();
        __syncthreads();
        for (int32_t i = i0; i < i1; ++i) {
            const int32_t blk = tile.block(i);
            const int buf = (i - i0) & 1;
            const int32_t blk1 = tile.block(min(i + 1, i1 - 1));
            next = valid_pages(p, tile, blk1, next);
            if (i + 1 < i1) stage(p, blk1, next, wave, lds + (buf ^ 1) * kStage<KS, ND>);
            const int32_t after = load_pages(p, tile, tile.block(min(i + 2, i1 - 1)));
            const FromLds<KS, ND> src{lds + buf * kStage<KS, ND> + lane * 16};
            attend_block<KS, ND>(p, table, st, src, pages, blk, row.sees, tile.full(p, blk));
            pages = next;
            next = after;
            wait_staged();
            __syncthreads();
        }
    }
    if (!row.have) return;
    if (p.splits > 1) {
        const int64_t at = (row.t * p.H + row.head) * p.splits + split;
        if (g == 0) {
            p.mz[2 * at] = (double)st.m;
            p.mz[2 * at + 1] = st.z;
        }
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            if (16 * dt >= p.kv.D) break;
            double* s = p.sums + at * p.kv.D + 16 * dt + 4 * g;
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = st.acc[dt][i];
        }
        return;
    }
    const double unit = out_unit(p, st.z);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        if (16 * dt >= p.kv.D) break;
        int32_t q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = out_code(p, st.acc[dt][i], st.z, unit);
        const int32_t d = 16 * dt + 4 * g;
        const int64_t at = row.t * p.ldy + (int64_t)row.head * p.kv.D + d;
        if (!p.vec_y) {
#pragma unroll
            for (int i = 0; i < 4; ++i) store_out(p, row.t, row.head, d + i, q[i]);
        } else if (p.out_bits == 8) {
            *reinterpret_cast<uint32_t*>(static_cast<int8_t*>(p.y) + at) =
                (uint32_t)(uint8_t)q[0] | ((uint32_t)(uint8_t)q[1] << 8) |
                ((uint32_t)(uint8_t)q[2] << 16) | ((uint32_t)(uint8_t)q[3] << 24);
        } else {
            *reinterpret_cast<uint2*>(static_cast<int16_t*>(p.y) + at) =
                make_uint2((uint32_t)(uint16_t)q[0] | ((uint32_t)(uint16_t)q[1] << 16),
                           (uint32_t)(uint16_t)q[2] | ((uint32_t)(uint16_t)q[3] << 16));
        }
    }
}

// The split's blocks [i0, i1) of the tile.
__device__ inline void split_range(const AttnArgs& p, const Tile& t, int split, int32_t& i0,
                                   int32_t& i1)
{
    const int32_t per = (t.n + p.splits - 1) / p.splits;
    i0 = per * split;
    i1 = min(i0 + per, t.n);
}

// grid (tiles of 16 rows, G, splits)
template <int KS, int ND>
__global__ __launch_bounds__(256, KS == 1 ? 3 : KS == 2 ? 2 : 1) void paged_attn_split_kernel(AttnArgs p)
{
    constexpr int J = ND < 4 ? ND : 4;
    __shared__ double lds[kJoinDoubles<J>];
    Tile tile;
    if (!find_tile<kRows>(p, blockIdx.x, tile)) return;
    int32_t i0, i1;
    split_range(p, tile, blockIdx.z, i0, i1);
    split_rows<KS, ND, J>(p, tile, blockIdx.y, i0, i1, blockIdx.z, lds);
}

// Work-groups go to the eight XCDs in turn, each with an L2 of its own: those
// that read the same keys (a cache head's part) are given to one XCD, or to
// 8 / n of them in turn where there are n < 8 such parts.  The tiles of an
// XCD come heaviest first up to the middle (the last tokens of a prompt see
// the most keys), then lightest first, so that a CU's two work-groups add up
// to the same.
struct Place {
    int64_t tile;
    int32_t part;  // g + G * split
};
__device__ inline Place place_of(const AttnArgs& p, int64_t id, int64_t tiles)
{
    const int64_t parts = (int64_t)p.kv.G * p.splits;
    Place w;
    int64_t n = tiles, at;
    if (parts % 8 == 0) {
        const int64_t slot = id >> 3;
        w.part = (int32_t)((slot / tiles) * 8 + (id & 7));
        at = slot % tiles;
    } else if (8 % parts == 0) {
        const int64_t r = 8 / parts;
        w.part = (int32_t)((id & 7) % parts);
        n = (tiles + r - 1) / r;
        at = id >> 3;
        w.tile = ((id & 7) / parts);  // of every r tiles
        at = at < n - n / 2 ? n - 1 - at : at - (n - n / 2);
        w.tile += at * r;
        return w;
    } else {
        w.part = (int32_t)(id / tiles);
        at = id % tiles;
    }
    w.tile = at < n - n / 2 ? n - 1 - at : at - (n - n / 2);
    return w;
}

// One work-group per tile of 64 rows, cache head and split; a sequence's last
// 16 rows or fewer are split among the waves.
template <int KS, int ND>
__global__ __launch_bounds__(256, KS == 1 ? 3 : KS == 2 ? 2 : 1) void paged_attn_tile_kernel(AttnArgs p,
                                                                               int64_t tiles)
{
    __shared__ __attribute__((aligned(1024))) int8_t lds[2 * kStage<KS, ND>];
    const Place w = place_of(p, blockIdx.x, tiles);
    const int32_t g0 = w.part % p.kv.G, split = w.part / p.kv.G;
    Tile tile;
    if (w.tile >= tiles || !find_tile<kTile>(p, w.tile, tile)) return;
    int32_t i0, i1;
    split_range(p, tile, split, i0, i1);
    if (tile.rows - tile.row0 <= kRows)
        split_rows<KS, ND, 1>(p, tile, g0, i0, i1, split, reinterpret_cast<double*>(lds));
    else
        share_keys<KS, ND>(p, tile, g0, i0, i1, split, (MQ_LDS int8_t*)lds);
}

// Joins the splits: NW waves per row and 64 channels, each every NW-th split
// (up to 8, 64 or all of them).  Latency bounds it: the first eight sums are
// read before the maxima they are weighed by are looked at.
template <int NW>
__global__ __launch_bounds__(NW < 4 ? 256 : 64 * NW) void paged_attn_join_kernel(AttnArgs p)
{
    __shared__ double lds[NW][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int units = NW < 4 ? 4 / NW : 1;
    constexpr int slots = NW < 16 ? 1 : kMaxSplits / 64;  // of 64 splits
    const int64_t row = (int64_t)blockIdx.x * units + wave / NW;
    if (row >= p.T * p.H) return;
    const int w = wave % NW;
    const int32_t d = blockIdx.y * 64 + lane;
    const bool have = d < p.kv.D;
    const double* x = p.sums + row * p.splits * p.kv.D + (have ? d : 0);
    const double* mz = p.mz + row * p.splits * 2;
    double v[8], m[slots], f[slots], zs[slots];
    auto load = [&](int i, int s0) {
        const int end = min(64, p.splits - 64 * i);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (s0 + u * NW < end) v[u] = x[(int64_t)(64 * i + s0 + u * NW) * p.kv.D];
    };
#pragma unroll
    for (int i = 0; i < slots; ++i) {
        const int s = min(lane + 64 * i, p.splits - 1);
        m[i] = mz[2 * s];
        zs[i] = mz[2 * s + 1];
    }
    load(0, w);
    const int64_t t = row / p.H;
    if (t < p.kv.starts[0] || t >= p.kv.starts[p.kv.B]) return;  // rows of no sequence
    double top = m[0], z = 0.0;
#pragma unroll
    for (int i = 1; i < slots; ++i) top = fmax(top, m[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmax(top, __shfl_xor(top, o));
#pragma unroll
    for (int i = 0; i < slots; ++i) {
        f[i] = exp2_poly(fmax(-p.tau * (top - m[i]), -1000.0));
        if (lane + 64 * i < p.splits) z = __builtin_fma(f[i], zs[i], z);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) z += __shfl_xor(z, o);
    double acc = 0.0;
#pragma unroll
    for (int i = 0; i < slots; ++i) {
        const int end = min(64, p.splits - 64 * i);
        for (int s0 = w; s0 < end; s0 += 8 * NW) {
            if (i > 0 || s0 > w) load(i, s0);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (s0 + u * NW < end)
                    acc = __builtin_fma(__shfl(f[i], s0 + u * NW), v[u], acc);
        }
    }
    if (NW > 1) {
        lds[wave][lane] = acc;
        __syncthreads();
        if (w != 0) return;
        acc = 0.0;
#pragma unroll
        for (int i = 0; i < NW; ++i) acc += lds[i][lane];
    }
    if (have) store_out(p, t, (int32_t)(row % p.H), d, out_code(p, acc, z, out_unit(p, z)));
}

// Row tiles of all sequences, at most.
int64_t row_tiles(int64_t T, int64_t B, int32_t grp, int R) { return T * grp / R + B; }

// Whether the sequences have more rows than a wave takes, on average.
bool tiled(int64_t T, int64_t B, int32_t grp) { return T * grp > B * kRows; }

// Parts the keys of every tile are split into: as many work-groups as the chip
// holds at once, at least a block per wave in each.  With fewer or more (us,
// main kernel): 64 sequences up to 4096 keys, 4 heads of 64, 256 work-groups
// 35, 512 23, 768 27, 1024 28; 2 up to 120000, one head of 256: 64 work-groups
// 41, 256 28, 470 36.
int64_t split_count(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D, int64_t max_len)
{
    const int32_t grp = H / G;
    const int R = tiled(T, B, grp) ? kTile : kRows;
    const int64_t groups = std::max(T * grp / R, std::min(B, T)) * G;
    // two work-groups per CU fit, one where the state is large (D > 128)
    int64_t s = (D > 128 ? 256 : 512) / std::max<int64_t>(groups, 1);
    const int64_t blocks = (max_len + kBlk - 1) / kBlk;
    s = std::min(s, (blocks + kWaves - 1) / kWaves);
    s = std::min<int64_t>(s, MQ_ATTN_MAX_WORKSPACE / (T * H * (D + 2) * 8));
    return std::max<int64_t>(1, std::min<int64_t>(s, kMaxSplits));
}

template <int ND>
hipError_t launch_main(const AttnArgs& p, int64_t B, hipStream_t s)
{
    constexpr int KS = (ND + 3) / 4;
    const int64_t parts = (int64_t)p.kv.G * p.splits;
    if (tiled(p.T, B, p.grp)) {
        const int64_t tiles = row_tiles(p.T, B, p.grp, kTile);
        // (see place_of)
        const int64_t n = parts % 8 != 0 && 8 % parts == 0
                              ? 8 * ((tiles + 8 / parts - 1) / (8 / parts))
                              : tiles * parts;
        if (n >= kMaxBlocks) return hipErrorInvalidConfiguration;
        paged_attn_tile_kernel<KS, ND><<<(unsigned)n, 256, 0, s>>>(p, tiles);
        return hipGetLastError();
    }
    const int64_t n = row_tiles(p.T, B, p.grp, kRows);
    if (n >= kMaxBlocks) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)n, (unsigned)p.kv.G, (unsigned)p.splits);
    paged_attn_split_kernel<KS, ND><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace

int64_t paged_attn_workspace(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D, int64_t max_len)
{
    if (T == 0 || B == 0) return 0;
    const int64_t s = split_count(T, B, H, G, D, max_len);
    return s > 1 ? s * T * H * (D + 2) * 8 : 0;
}

hipError_t launch_paged_attn(const KvArgs& kv, const int16_t* q, int64_t ldq, int64_t T, int32_t H,
                             float q_scale, int32_t q_zp, float k_scale, float v_scale,
                             int32_t v_zp, float logit_scale, int64_t window, int64_t sinks,
                             float out_scale, int32_t out_zp, int32_t out_bits, void* y,
                             int64_t ldy, int64_t max_len, void* ws, int64_t ws_bytes,
                             hipStream_t s)
{
    AttnArgs p;
    p.kv = kv;
    if (kv.pages == 0) p.kv.ld = 0;  // no place: no block is looked at
    p.q = q;
    p.y = y;
    p.ldq = ldq;
    p.ldy = ldy;
    p.T = T;
    p.H = H;
    p.grp = H / kv.G;
    p.q_zp = q_zp;
    p.v_zp = v_zp;
    p.out_zp = out_zp;
    p.out_bits = out_bits;
    const double sigma = (double)q_scale * (double)k_scale * (double)logit_scale;
    // (from 128 on only the largest logits of a block, and of the row, weigh
    // anything, whatever the scale)
    p.tau = std::min(sigma * 1.4426950408889634, 128.0);  // log2(e)
    p.v_scale = v_scale;
    p.out_scale = out_scale;
    // a weight is 0 below 1/2: from 2^-40 of the largest on whatever the
    // distance (tau d_cut <= 40 + tau)
    const double cut = 40.0 / p.tau;
    p.d_cut = cut < 4294967295.0 ? (uint32_t)std::ceil(cut) : 0xFFFFFFFFu;
    // positions are below 2^31: a window of as many hides nothing
    p.window = window < 0x7FFFFFFF ? (int32_t)window : 0;
    p.sinks = p.window > 0 ? (int32_t)std::min<int64_t>(sinks, 0x7FFFFFFF) : 0;
    p.page_bytes = (kv.G * kv.D) << kv.shift;
    p.vec_q = ((uintptr_t)q % 16) == 0 && ldq % 8 == 0;
    p.vec_y = ((uintptr_t)y % (out_bits / 2)) == 0 && ldy % 4 == 0;
    // the blocks that a row of a windowed call walks over
    if (window > 0 && window < max_len)
        max_len = std::min(max_len, window + std::min<int64_t>(p.sinks, max_len) + 2 * kBlk);
    int64_t splits = split_count(T, kv.B, H, kv.G, kv.D, max_len);
    const int64_t one = T * H * (kv.D + 2) * 8;
    splits = ws ? std::min(splits, std::max<int64_t>(ws_bytes / one, 1)) : 1;
    p.splits = (int32_t)splits;
    p.mz = static_cast<double*>(ws);
    p.sums = p.mz + T * H * splits * 2;
    hipError_t e;
    switch ((kv.D + 31) / 32) {
    case 1: e = launch_main<2>(p, kv.B, s); break;
    case 2: e = launch_main<4>(p, kv.B, s); break;
    case 3: e = launch_main<6>(p, kv.B, s); break;
    case 4: e = launch_main<8>(p, kv.B, s); break;
    case 5: e = launch_main<10>(p, kv.B, s); break;
    case 6: e = launch_main<12>(p, kv.B, s); break;
    case 7: e = launch_main<14>(p, kv.B, s); break;
    default: e = launch_main<16>(p, kv.B, s); break;
    }
    if (e != hipSuccess || splits == 1) return e;
    const unsigned chunks = (unsigned)((kv.D + 63) / 64);
    const int64_t rows = T * H;
    if (splits <= 8)
        paged_attn_join_kernel<1><<<dim3((unsigned)((rows + 3) / 4), chunks), 256, 0, s>>>(p);
    else if (splits <= 64)
        paged_attn_join_kernel<4><<<dim3((unsigned)rows, chunks), 256, 0, s>>>(p);
    else
        paged_attn_join_kernel<16><<<dim3((unsigned)rows, chunks), 1024, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mq
