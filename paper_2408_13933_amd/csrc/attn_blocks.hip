// Attention of new tokens over the cache with block scales, in one pass with a
// running maximum, scores and weights in registers throughout.
//
// A wave holds 16 rows (a row: one token's query head; the H / G heads that
// share a cache head lie next to each other) per set and walks over blocks of 64
// key positions.  Both products run on the fp16 matrix instructions with fp32
// sums: codes are exact in fp16, the queries of a row are scaled by a power of
// two to below 2^15, which leaves those of 16 bits exact down to 2^-31 of the row's
// largest (below, as for all, a step is 2^-24), fp32 ones as the sum of two fp16
// numbers (22 bits).  Scores come out transposed,
//   C[key][row] = K[key][d] * Q[row][d],
// a lane holding one row (lane & 15) and, the 16 keys of tile j being taken in
// the order 16 (r >> 2) + 4 j + (r & 3), the 16 consecutive keys of one group: the
// layout that the second product takes as its operand,
//   O[d][row] = V^T[d][key] * W[key][row].
// The keys of a lane share their block's scales.  The key scale joins the factor
// of the logits; the value scale joins the exponent, so that the weights
// 2^(x + log2 vs - m) multiply bare codes, and the sum of the softmax takes a
// lane's weights by 1 / vs once per 16 keys.  The running maximum m is that of x +
// log2 vs; it moves only when exceeded by 2^7, so weights stay below 2^15.
// Weights are rounded to fp16 (11 bits, the outputs have 8 or 11), for fp32
// outputs to the sum of two (500 tokens over 16000: 285 us with two terms of queries
// and weights, 160 with one); statistics and outputs are fp32.  Contexts of windows of 1000
// keys are 2.7e-4 off in fp16, of which their own rounding makes 2.0e-4.
#include <algorithm>
#include <cmath>

#include "kvblocks.h"
#include "kvwalk.h"
#include "mq_internal.h"
#include "tokens.h"
#include "wave.h"

#define MQ_LDS __attribute__((address_space(3)))
#define MQ_GLOBAL __attribute__((address_space(1)))

namespace mq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr int kBlk = 64;                  // key positions per step
constexpr int kRows = 16;                 // rows per set
constexpr int kWaves = 4;                 // waves per work-group that share keys
constexpr int kTile = 32 * kWaves;        // rows per work-group where the waves share keys
constexpr int kMaxParts = 512;
// sequences of a call whose parts are planned on the device, 64 per lane register
constexpr int kPlanRegs = 4, kPlanned = 64 * kPlanRegs;
constexpr float kNone = -0x1.fffffep127f; // running maximum of a row that has seen nothing
constexpr float kTop = 8.0f, kLag = 7.0f; // weights up to 2^(kTop + kLag)
constexpr float kHuge = 0x1p21f;          // maxima from here on: far_exponent
using Tile = RowTile<kBlk>;

struct AttnArgs {
    KvArgs kv;
    const float* k_scale;
    const float* v_scale;
    int32_t bshift;
    int32_t type;
    const void* q;
    void* y;
    int64_t ldq, ldy, T;
    int32_t H, grp;        // grp = H / G
    float tau;             // log2(e) * logit_scale
    int32_t window, sinks; // window 0: none
    int32_t page_bytes;    // of a page's keys, and of its values (at most 2^28)
    int32_t vec_q, vec_y;  // query rows in 16-byte chunks, output rows in fours of elements
    int32_t splits;        // of every tile of rows that share keys
    int32_t target;        // work-groups to plan the rows' parts for; 0: one part each
    int32_t slots;         // work-groups of such rows per head
    // sums of weights times codes, maximum and weight sum of a part: [row][split] of
    // tiles, [head][work-group][16 rows] of planned parts
    float* sums;           // [][D]
    float* ml;             // [][2]
};

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline v4f mfma(v8h a, v8h b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight codes as fp16, exact: the byte c + 128 in the low bits of 1024 is 1152 + c.
__device__ inline v8h to_half(int32_t x, int32_t y)
{
    const v2h off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
    const uint32_t b[2] = {(uint32_t)x ^ 0x80808080u, (uint32_t)y ^ 0x80808080u};
    v8h h;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const v2h lo =
            __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, b[i], 0x04010400u)) + off;
        const v2h hi =
            __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, b[i], 0x04030402u)) + off;
        h[4 * i] = lo[0];
        h[4 * i + 1] = lo[1];
        h[4 * i + 2] = hi[0];
        h[4 * i + 3] = hi[1];
    }
    return h;
}
__device__ inline void to_half(const v4i& x, v8h (&h)[2])
{
    h[0] = to_half(x[0], x[1]);
    h[1] = to_half(x[2], x[3]);
}

// Over the four lanes of a row.
__device__ inline uint32_t swap16(uint32_t v, uint32_t& o)
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    o = a[1];
    return a[0];
}
__device__ inline uint32_t swap32(uint32_t v, uint32_t& o)
{
    const auto a = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    o = a[1];
    return a[0];
}
template <class F>
__device__ inline float over_row(float v, F f)
{
    uint32_t o;
    uint32_t a = swap16(__builtin_bit_cast(uint32_t, v), o);
    v = f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, o));
    a = swap32(__builtin_bit_cast(uint32_t, v), o);
    return f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, o));
}
__device__ inline float row_max(float v)
{
    return over_row(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ inline float row_sum(float v)
{
    return over_row(v, [](float a, float b) { return a + b; });
}

// A set of 16 rows: KS steps of 64 channels (the last one of 32 where the number of 32
// is odd), ND tiles of 16 output channels, N fp16 terms of queries and of weights.
template <int KS, int ND, int N>
struct Rows {
    v8h q[N][KS][2];
    float a;         // of the products, in units of log2
    v4f acc[ND];     // output channels 16 dt + 4 (lane >> 4) + i of row lane & 15
    float m, l;      // l: this lane's keys only
    __device__ void clear()
    {
        m = kNone;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) acc[dt] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    }
};

// A row's queries from bits of its largest magnitude: times a power of two, as N
// fp16 terms; returns the factor of its products, in units of log2.  2^e <= most <
// 2^(e + 1): the row times 2^(14 - e).  A row that is not finite becomes NaN
// throughout.
struct Scaled {
    float up, a;
    __device__ Scaled(const AttnArgs& p, uint32_t most)
    {
        const uint32_t e = min(max(most >> 23, 27u), 254u);
        up = most < kInfBits ? __builtin_bit_cast(float, (268u - e) << 23) : __builtin_nanf("");
        a = p.tau * __builtin_bit_cast(float, (e - 14u) << 23);
    }
};
// Eight consecutive queries as they lie in memory (N == 2: fp32, else 16 bits).  One
// form for both types of 16 bits, which are told apart when they become numbers: a load
// and a conversion per type made three quarters of a kernel of 160 KB.
typedef unsigned short v2us __attribute__((ext_vector_type(2)));
template <int N>
struct Eight {
    uint32_t d[4 * N];
    __device__ void load(const AttnArgs& p, int64_t i)
    {
        if (p.vec_q) {
            const uint4* x = reinterpret_cast<const uint4*>(static_cast<const int8_t*>(p.q) +
                                                            i * (2 * N));
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const uint4 v = x[j];
                d[4 * j] = v.x, d[4 * j + 1] = v.y, d[4 * j + 2] = v.z, d[4 * j + 3] = v.w;
            }
        } else if constexpr (N == 2) {
#pragma unroll
            for (int j = 0; j < 8; ++j) d[j] = static_cast<const uint32_t*>(p.q)[i + j];
        } else {
            const uint16_t* x = static_cast<const uint16_t*>(p.q) + i;
#pragma unroll
            for (int j = 0; j < 4; ++j) d[j] = x[2 * j] | (uint32_t)x[2 * j + 1] << 16;
        }
    }
    __device__ void keep(bool have)
    {
#pragma unroll
        for (int j = 0; j < 4 * N; ++j) d[j] = have ? d[j] : 0;
    }
    // Magnitudes as bits, NaN and infinities the largest: of two numbers of 16 bits in one.
    __device__ uint32_t most(uint32_t m) const
    {
#pragma unroll
        for (int j = 0; j < 4 * N; ++j) {
            if constexpr (N == 2)
                m = max(m, d[j] & 0x7fffffffu);
            else
                m = __builtin_bit_cast(
                    uint32_t, __builtin_elementwise_max(__builtin_bit_cast(v2us, m),
                                                        __builtin_bit_cast(v2us, d[j] & 0x7fff7fffu)));
        }
        return m;
    }
    // Bits of the fp32 number of what `most` found.
    static __device__ uint32_t bits(const AttnArgs& p, uint32_t m)
    {
        if constexpr (N == 2) return m;
        m = max(m & 0xffffu, m >> 16);
        return p.type == MQ_BF16 ? m << 16
                                 : __builtin_bit_cast(
                                       uint32_t, (float)__builtin_bit_cast(_Float16, (uint16_t)m));
    }
    // Times `up`, as N fp16 terms.
    __device__ void terms(const AttnArgs& p, float up, v8h& a, v8h* b) const
    {
        auto put = [&](auto number) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float v = number(j) * up;
                const _Float16 h = (_Float16)v;
                a[j] = h;
                if constexpr (N == 2) (*b)[j] = (_Float16)(v - (float)h);
            }
        };
        if constexpr (N == 2)
            put([&](int j) { return __builtin_bit_cast(float, d[j]); });
        else if (p.type == MQ_BF16)
            put([&](int j) { return half_of<MQ_BF16>(d[j >> 1], j & 1); });
        else
            put([&](int j) { return half_of<MQ_F16>(d[j >> 1], j & 1); });
    }
};

// The first channel of a lane's eight of operand (s, h) of a set's products.
template <int ND>
__device__ inline int operand_channel(int s, int h)
{
    constexpr int KS = (ND + 3) / 4;
    const int g = (threadIdx.x & 63) >> 4;
    return (ND / 2) % 2 == 1 && s == KS - 1 ? 64 * s + 8 * g : 64 * s + 16 * g + 8 * h;
}
// Operands of step s.
template <int ND>
constexpr int halves(int s)
{
    return (ND / 2) % 2 == 1 && s == (ND + 3) / 4 - 1 ? 1 : 2;
}

// Channels past the head and rows past the tile are 0.  All lanes read (those the row's
// first channels; a row past the tile is its last one): where loads depended on the lane,
// the compiler (HIP 7.2) moved registers of all lanes to accumulators with part of the
// lanes off, and lost what the others held.
template <int KS, int ND, int N>
__device__ inline void load_queries(const AttnArgs& p, const RowAt& row, Rows<KS, ND, N>& st)
{
    const int64_t at = row.t * p.ldq + (int64_t)row.head * p.kv.D;
    Eight<N> x[KS][2];
    uint32_t most = 0;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < halves<ND>(s); ++h) {
            const int d = operand_channel<ND>(s, h);
            const bool have = row.have && d < p.kv.D;
            x[s][h].load(p, at + (have ? d : 0));
            x[s][h].keep(have);
            most = x[s][h].most(most);
        }
    uint32_t o;
    most = swap16(Eight<N>::bits(p, most), o);
    most = max(most, o);
    most = swap32(most, o);
    most = max(most, o);
    const Scaled sc(p, most);
    st.a = sc.a;
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int h = 0; h < halves<ND>(s); ++h)
            x[s][h].terms(p, sc.up, st.q[0][s][h], &st.q[N - 1][s][h]);
}
// The same for 32 rows: channels 32 u + 16 (lane >> 5) on; in two passes over fp32 rows,
// whose channels do not all fit beside the rest.
template <int DT, int N>
__device__ inline float load_queries32(const AttnArgs& p, const RowAt& row, v8h (&q)[N][DT][2])
{
    const int hh = (threadIdx.x & 63) >> 5;
    const int64_t at = row.t * p.ldq + (int64_t)row.head * p.kv.D;
    Eight<N> x[N == 2 ? 1 : DT][2];
    uint32_t most = 0;
    auto read = [&](int u, Eight<N> (&e)[2]) {
        const int d = 32 * u + 16 * hh;
        const bool have = row.have && d < p.kv.D;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            e[h].load(p, at + (have ? d : 0) + 8 * h);
            e[h].keep(have);
        }
    };
#pragma unroll
    for (int u = 0; u < DT; ++u) {
        read(u, x[N == 2 ? 0 : u]);
#pragma unroll
        for (int h = 0; h < 2; ++h) most = x[N == 2 ? 0 : u][h].most(most);
    }
    uint32_t o;
    most = swap32(Eight<N>::bits(p, most), o);
    most = max(most, o);
    const Scaled sc(p, most);
#pragma unroll
    for (int u = 0; u < DT; ++u) {
        if constexpr (N == 2) read(u, x[0]);
#pragma unroll
        for (int h = 0; h < 2; ++h)
            x[N == 2 ? 0 : u][h].terms(p, sc.up, q[0][u][h], &q[N - 1][u][h]);
    }
    return sc.a;
}

// Where a lane reads a block: keys 16 (r >> 2) + (r & 3) of tile 0 (tile j: 4 j rows
// on) from channel 16 g on, and 16 values of channel r of group g.
struct Spot {
    int32_t key, value;  // page list entry's offset (in 16-position groups) of the lane
    __device__ Spot()
    {
        const int lane = threadIdx.x & 63;
        key = (lane & 15) >> 2;
        value = lane >> 4;
    }
};
// Page list entries of a lane's two groups of a block, as they are.
struct Pages {
    int32_t key, value;
};
__device__ inline int32_t entry_of(const AttnArgs& p, int32_t blk, int32_t group)
{
    return (blk * kBlk + 16 * group) >> p.kv.shift;
}
__device__ inline Pages load_pages(const AttnArgs& p, const Tile& t, int32_t blk)
{
    const Spot s;
    const int32_t* list = p.kv.table + (int64_t)t.b * p.kv.ld;
    return Pages{list[min(entry_of(p, blk, s.key), t.last)],
                 list[min(entry_of(p, blk, s.value), t.last)]};
}
__device__ inline bool is_page(const AttnArgs& p, const Tile& t, int32_t blk, int32_t group,
                               int32_t page)
{
    return entry_of(p, blk, group) <= t.last && page >= 0 && page < (int32_t)p.kv.pages;
}

// A block's addresses for this lane; groups without a place read page 0's.
struct Addr {
    const MQ_GLOBAL int8_t* k;
    const MQ_GLOBAL int8_t* v;
    uint64_t scale;
    bool placed;  // the value group
    __device__ Addr(const AttnArgs& p, const Tile& t, int32_t g0, int32_t blk, const Pages& pg)
    {
        const Spot s;
        const uint32_t lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
        const uint32_t mask = (1u << p.kv.shift) - 1, D = (uint32_t)p.kv.D;
        const uint32_t kp = is_page(p, t, blk, s.key, pg.key) ? (uint32_t)pg.key : 0;
        placed = is_page(p, t, blk, s.value, pg.value);
        const uint32_t vp = placed ? (uint32_t)pg.value : 0;
        // in a page, whose bytes are at most 2^28 (the head's part uniform)
        const uint32_t head = (uint32_t)g0 << p.kv.shift;
        const uint32_t ks = (blk * kBlk + 16 * s.key) & mask, vs = (blk * kBlk + 16 * s.value) & mask;
        k = (const MQ_GLOBAL int8_t*)p.kv.k +
            ((uint64_t)kp * (uint32_t)p.page_bytes + (head * D + (ks + (r & 3)) * D + 16 * g));
        v = (const MQ_GLOBAL int8_t*)p.kv.v +
            ((uint64_t)vp * (uint32_t)p.page_bytes + (head * D + vs * D + 16 * r));
        scale = (uint64_t)vp * ((uint32_t)p.kv.G << (p.kv.shift - p.bshift)) +
                ((head + vs) >> p.bshift);
    }
};

// Channels past the head dimension: the scores read the head's first ones again
// (the queries are 0 there), the outputs of such a tile are dropped.  Offset of a
// lane's channels of step s from its first address (channel 16 g).
template <int ND>
__device__ inline int32_t key_chunk(const AttnArgs& p, int s)
{
    const int32_t d = operand_channel<ND>(s, 0), c = 16 * (((int)threadIdx.x & 63) >> 4);
    return (d < p.kv.D ? d : 0) - c;
}

// How 16 scores of a lane become weights, 2^(a c + b); lv, iv: log2 and inverse of
// the value scale.
struct Weigh {
    float a, b, lv, iv;
    // what the row's running maximum has to be compared with
    __device__ float top(float row_a, float ks, float vs, float most)
    {
        // (not 0: a product with -infinity stays that)
        a = fmaxf(row_a * ks, 0x1p-126f);
        lv = __builtin_amdgcn_logf(vs);
        iv = exp2_fast(-lv);
        return __builtin_fmaf(most, a, lv);
    }
};

// Exponent of a weight in a wave with rows whose maximum's last place is as large as a
// weight's range.  Theirs comes from the very number that the maximum was taken over, so
// that the largest weight is 2^kTop up to 2^(kTop + kLag) there too.  (By f.b the two differ
// by half a last place of the maximum, which from 2^29 on left fp16 nothing of any weight.)
// The other rows keep their bits.
__device__ inline float far_exponent(const Weigh& f, float score, float m)
{
    return fabsf(m) >= kHuge ? (__builtin_fmaf(score, f.a, f.lv) - m) + kTop
                             : __builtin_fmaf(score, f.a, f.b);
}

// Scores of 16 consecutive keys from `first` on that the row does not see (or that
// have no place) become -infinity.  Scales of a group without any are 1 (they may be
// anything there).
template <class Get>
__device__ inline void mask_scores(const AttnArgs& p, const Sees& sees, int32_t first, bool placed,
                                   float& ks, float& vs, Get score)
{
    // of the 16 keys on those below x, as bits
    auto below = [&](int32_t x) { return (1u << max(min(x - first, 16), 0)) - 1; };
    uint32_t seen = below(sees.hi + 1) & (~below(sees.lo + 1) | below(p.sinks));
    if (!placed) seen = 0;
    if (seen == 0) ks = vs = 1.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int keep = __builtin_amdgcn_sbfe((int)seen, i, 1);  // all ones or 0
        const float y = score(i);
        const int x = __builtin_bit_cast(int, y);
        score(i, __builtin_bit_cast(float, (x & keep) | ((int)0xff800000u & ~keep)));
    }
}

// Weight i (of 8 of an operand) as N fp16 numbers; sum: of the lane's, not of the
// rounded ones (a weight by a small value scale may be below fp16 and still count
// there).
template <int N>
__device__ inline void weigh(const Weigh& f, float score, int i, v8h (&w)[N], float& sum)
{
    const float x = exp2_fast(__builtin_fmaf(score, f.a, f.b));
    const _Float16 h = (_Float16)x;
    w[0][i] = h;
    if constexpr (N == 2) w[1][i] = (_Float16)(x - (float)h);
    sum += x;
}

// Least value scale that is told apart (its inverse times weights stays finite).
__device__ inline float value_scale(float vs) { return fmaxf(vs, 0x1p-67f); }

// 1 / l; 0 for a row that sees nothing.
__device__ inline float out_unit(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// Element of a row's first output, and four outputs from channel d on (N == 2: fp32).
__device__ inline int64_t out_at(const AttnArgs& p, int64_t t, int32_t head)
{
    return t * p.ldy + (int64_t)head * p.kv.D;
}
template <int N>
__device__ inline void store_four(const AttnArgs& p, int64_t row, int32_t d, v4f v)
{
    if constexpr (N == 2) {
        float* y = static_cast<float*>(p.y) + row + d;
        if (p.vec_y) {
            *reinterpret_cast<v4f*>(y) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = v[i];
        }
    } else {
        uint16_t* y = static_cast<uint16_t*>(p.y) + row + d;
        uint32_t h[2];
        if (p.type == MQ_BF16) {
            h[0] = pack2<MQ_BF16>(v[0], v[1]);
            h[1] = pack2<MQ_BF16>(v[2], v[3]);
        } else {
            h[0] = pack2<MQ_F16>(v[0], v[1]);
            h[1] = pack2<MQ_F16>(v[2], v[3]);
        }
        if (p.vec_y) {
            *reinterpret_cast<uint2*>(y) = make_uint2(h[0], h[1]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (uint16_t)(h[i >> 1] >> (16 * (i & 1)));
        }
    }
}
__device__ inline void store_four(const AttnArgs& p, int64_t row, int32_t d, v4f v)
{
    if (p.type == MQ_F32) store_four<2>(p, row, d, v);
    else store_four<1>(p, row, d, v);
}

// Where a part's state goes: sums + at D and ml + 2 at, row r's 16 rows on; or,
// of a row's only part, to the outputs.
struct PartAt {
    bool only;
    int64_t at;
};

// W waves share 16 rows and take every W-th block of [i0, i1), straight from
// the cache; their states are joined through LDS.
template <int ND, int W>
constexpr int kJoinFloats = W * (4 * ND * 64 + 2 * kRows);
template <int KS, int ND, int N, int W>
__device__ inline void split_rows(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, const RowAt& row, PartAt part, float* lds)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Rows<KS, ND, N> st;
    st.clear();
    int32_t i = i0 + wave;
    if (i < i1) {
        Pages pg = load_pages(p, tile, tile.block(i));
        load_queries(p, row, st);
        // values are read a block ahead; keys too where there are registers for them,
        // else once the block before has its scores
        constexpr bool kAhead = KS <= 2;
        struct Block {
            v4i k[4][KS], v[ND];
            float ks, vs;
            bool placed;
        };
        Block buf[2];
        Addr at(p, tile, g0, tile.block(i), pg);
        auto read_keys = [&](Block& x) {
            x.ks = p.k_scale[at.scale];
            x.vs = p.v_scale[at.scale];
            x.placed = at.placed;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const MQ_GLOBAL int8_t* from = at.k + (4 * j * p.kv.D + key_chunk<ND>(p, s));
                    if (halves<ND>(s) == 2) {
                        x.k[j][s] = *reinterpret_cast<const MQ_GLOBAL v4i*>(from);
                    } else {
                        const v2i h = *reinterpret_cast<const MQ_GLOBAL v2i*>(from);
                        x.k[j][s] = v4i{h[0], h[1], 0, 0};
                    }
                }
        };
        auto read_values = [&](Block& x) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
                if (dt < ND - 1 || 16 * dt < p.kv.D)
                    x.v[dt] = *reinterpret_cast<const MQ_GLOBAL v4i*>(at.v + 256 * dt);
        };
        auto ahead = [&](int32_t x) { return tile.block(min(x, i1 - 1)); };
        read_keys(buf[0]);
        read_values(buf[0]);
        pg = load_pages(p, tile, ahead(i + W));
        auto block = [&](Block& now, Block& next) {
            const int32_t blk = tile.block(i);
            at = Addr(p, tile, g0, ahead(i + W), pg);
            pg = load_pages(p, tile, ahead(i + 2 * W));
            if constexpr (kAhead) read_keys(next);
            read_values(next);
            __builtin_amdgcn_sched_barrier(0);
            // (what is read without registers to spare goes into the keys just used)
            float ks = now.ks, vs = now.vs;
            const bool placed = now.placed;
            // scores of keys 16 g + 4 j + i
            v4f c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const v4i& x = (kAhead ? now : buf[0]).k[j][s];
#pragma unroll
                    for (int h = 0; h < halves<ND>(s); ++h) {
                        const v8h k = to_half(x[2 * h], x[2 * h + 1]);
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            c[j] = mfma(k, st.q[e][s][h],
                                        s + h + e ? c[j] : v4f{0.0f, 0.0f, 0.0f, 0.0f});
                    }
                }
            if constexpr (!kAhead) {
                read_keys(buf[0]);
                next.ks = buf[0].ks;
                next.vs = buf[0].vs;
                next.placed = buf[0].placed;
            }
            if (!tile.full(p, blk) || __ballot(!placed) != 0) {
                struct {
                    v4f (&c)[4];
                    __device__ float operator()(int i) const { return c[i >> 2][i & 3]; }
                    __device__ void operator()(int i, float x) const { c[i >> 2][i & 3] = x; }
                } score{c};
                mask_scores(p, row.sees, blk * kBlk + 16 * g, placed, ks, vs, score);
            }
            float m = c[0][0];
#pragma unroll
            for (int x = 1; x < 16; ++x) m = fmaxf(m, c[x >> 2][x & 3]);
            Weigh f;
            m = row_max(f.top(st.a, ks, value_scale(vs), m));
            if (__ballot(m - st.m > kLag) != 0) {  // (the sum could round up)
                m = fmaxf(m, st.m);
                const float down = exp2_fast(st.m - m);
                st.l *= down;
#pragma unroll
                for (int dt = 0; dt < ND; ++dt) st.acc[dt] *= down;
                st.m = m;
            }
            f.b = f.lv + (kTop - st.m);
            if (__ballot(fabsf(st.m) >= kHuge) != 0) {
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    c[x >> 2][x & 3] = far_exponent(f, c[x >> 2][x & 3], st.m);
                f.a = 1.0f;
                f.b = 0.0f;
            }
            v8h w[2][N];
            float sum = 0.0f;
#pragma unroll
            for (int x = 0; x < 16; ++x) weigh(f, c[x >> 2][x & 3], x & 7, w[x >> 3], sum);
            st.l = __builtin_fmaf(sum, f.iv, st.l);
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) {
                if (dt == ND - 1 && 16 * dt >= p.kv.D) break;
                v8h v[2];
                to_half(now.v[dt], v);
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < N; ++e) st.acc[dt] = mfma(v[h], w[h][e], st.acc[dt]);
            }
        };
        for (; i < i1; i += W) {
            block(buf[0], buf[1]);
            i += W;
            if (i >= i1) break;
            block(buf[1], buf[0]);
        }
    }
    float* lm = lds + W * 4 * ND * 64;  // [wave][row]
    float* ll = lm + W * kRows;
    const float l = row_sum(st.l);
    if (g == 0) {
        lm[wave * kRows + r] = st.m;
        ll[wave * kRows + r] = l;
    }
    v4f* acc = reinterpret_cast<v4f*>(lds);  // [wave][tile][lane]
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) acc[(wave * ND + dt) * 64 + lane] = st.acc[dt];
    __syncthreads();
    float m = kNone;
#pragma unroll
    for (int w = 0; w < W; ++w) m = fmaxf(m, lm[w * kRows + r]);
    float f[W], sum = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) {
        f[w] = exp2_fast(lm[w * kRows + r] - m);
        sum = __builtin_fmaf(f[w], ll[w * kRows + r], sum);
    }
    if (!row.have) return;
    if (!part.only && wave == 0 && g == 0) {
        p.ml[2 * part.at] = m;
        p.ml[2 * part.at + 1] = sum;
    }
    const float unit = out_unit(sum);
    const int64_t out = out_at(p, row.t, row.head);
#pragma unroll
    for (int i = 0; i < (ND + W - 1) / W; ++i) {
        const int dt = W * i + wave;
        const int32_t d = 16 * dt + 4 * g;
        if (16 * dt >= p.kv.D) break;
        v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const v4f x = acc[(w * ND + dt) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __builtin_fmaf(f[w], x[e], v[e]);
        }
        if (!part.only) *reinterpret_cast<v4f*>(p.sums + part.at * p.kv.D + d) = v;
        else store_four<N>(p, out, d, v * unit);
    }
}

// Where many rows share keys: a wave has 32 rows on the 32 x 32 x 16 instructions.
// Vector arithmetic (290 instructions a block, 32 of them exponentials) and products
// (32 of 32 cycles) add up: 500 tokens over 16000, 32 heads of 128 on 8, take 160 us
// and a join of 8, 0.77 PFLOP/s; two sets of 16 rows on the smaller instructions take the
// same, and so do the products of the next block's scores between this one's
// exponentials.
// Scores C[key][row] of 32 keys, the keys of tile t of a block in the order 32 t + 16
// ((r >> 2) & 1) + 4 (r >> 3) + (r & 3): a lane holds row lane & 31 and the 16
// consecutive keys of group 2 t + (lane >> 5), outputs in O[d][row].
struct Wide {
    int lane, r, hh;
    __device__ Wide()
    {
        lane = threadIdx.x & 63;
        r = lane & 31;
        hh = lane >> 5;
    }
};
typedef float v16f __attribute__((ext_vector_type(16)));
__device__ inline v16f mfma32(v8h a, v8h b, v16f c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// All four waves walk over blocks [i0, i1), whose codes they put into LDS as fp16, in
// the order of the lanes: keys (t, u) and values (t, u) of 32 channels u, two halves
// of 1 KB each.  A block's codes are read during the block before and converted once
// for all waves (by every wave for itself, with 16 rows each: 228 us instead of 170).
template <int DT>
constexpr int kStage = 4 * DT * 2048;
template <int DT, int N>
__device__ inline void share_keys(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, int split, MQ_LDS int8_t* lds)
{
    const Wide at;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowAt row(p, tile, tile.row0 + 32 * wave, g0, at.r);
    v16f acc[DT];
#pragma unroll
    for (int u = 0; u < DT; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[u][i] = 0.0f;
    float m = kNone, l = 0.0f;
    if (i0 < i1) {
        // waves 0 and 1 stage the keys of a tile, 2 and 3 the values
        const int t = wave & 1;
        const bool values = wave >= 2;
        const int32_t group = 2 * t + (values ? at.hh : (at.r >> 2) & 1);
        const uint32_t D = (uint32_t)p.kv.D, mask = (1u << p.kv.shift) - 1;
        // from the first slot of the group's 16: a key and its channels, or a
        // channel's 16 tokens; channels past the head read its first ones (queries are 0
        // there, such outputs are dropped)
        const uint32_t lane_at = values ? 16 * at.r : (4 * (at.r >> 3) + (at.r & 3)) * D + 16 * at.hh;
        const uint32_t step = values ? 512 : 32;
        const uint32_t last = (DT - 1) * step,
                       back = (values ? 32 * (DT - 1) + at.r : 32 * (DT - 1) + 16 * at.hh) < (int)D
                                  ? last
                                  : 0u - (values ? 16 * at.r : 16 * at.hh);
        const MQ_GLOBAL int8_t* const base =
            (const MQ_GLOBAL int8_t*)(values ? p.kv.v : p.kv.k) +
            (((uint32_t)g0 << p.kv.shift) * D + lane_at);
        const int32_t* const list = p.kv.table + (int64_t)tile.b * p.kv.ld;
        struct Entries {
            int32_t stage, scale[2];
        };
        auto entries = [&](int32_t i) {
            const int32_t blk = tile.block(min(i, i1 - 1));
            return Entries{list[min(entry_of(p, blk, group), tile.last)],
                           {list[min(entry_of(p, blk, at.hh), tile.last)],
                            list[min(entry_of(p, blk, 2 + at.hh), tile.last)]}};
        };
        struct Scales {
            float k[2], v[2];
            bool placed[2];
        };
        v4i raw[DT];
        Entries pg = entries(i0);
        auto read = [&](int32_t i, Scales& s) {
            const int32_t blk = tile.block(min(i, i1 - 1));
            const uint32_t page = is_page(p, tile, blk, group, pg.stage) ? (uint32_t)pg.stage : 0;
            const uint32_t slot = (uint32_t)(blk * kBlk + 16 * group) & mask;
            const MQ_GLOBAL int8_t* x = base + ((uint64_t)page * (uint32_t)p.page_bytes + slot * D);
#pragma unroll
            for (int u = 0; u < DT - 1; ++u)
                raw[u] = *reinterpret_cast<const MQ_GLOBAL v4i*>(x + u * step);
            raw[DT - 1] = *reinterpret_cast<const MQ_GLOBAL v4i*>(x + (int32_t)back);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int32_t g = 2 * j + at.hh;
                s.placed[j] = is_page(p, tile, blk, g, pg.scale[j]);
                const uint32_t sp = s.placed[j] ? (uint32_t)pg.scale[j] : 0;
                const uint64_t e =
                    (uint64_t)sp * ((uint32_t)p.kv.G << (p.kv.shift - p.bshift)) +
                    ((((uint32_t)g0 << p.kv.shift) + ((uint32_t)(blk * kBlk + 16 * g) & mask)) >>
                     p.bshift);
                s.k[j] = p.k_scale[e];
                s.v[j] = p.v_scale[e];
            }
            pg = entries(i + 1);
        };
        MQ_LDS int8_t* const mine = lds + ((values ? 2 : 0) + t) * DT * 2048 + at.lane * 16;
        auto put = [&](int buf) {
#pragma unroll
            for (int u = 0; u < DT; ++u) {
                v8h h[2];
                to_half(raw[u], h);
                MQ_LDS int8_t* to = mine + buf * kStage<DT> + u * 2048;
                *reinterpret_cast<MQ_LDS v8h*>(to) = h[0];
                *reinterpret_cast<MQ_LDS v8h*>(to + 1024) = h[1];
            }
        };
        // (fp32 rows of more than 224 channels leave no registers for the next block)
        constexpr bool kLate = DT == 8 && N == 2;
        Scales now, next;
        read(i0, now);
        v8h q[N][DT][2];
        const float qa = load_queries32<DT, N>(p, row, q);
        put(0);
        __syncthreads();
        for (int32_t i = i0; i < i1; ++i) {
            const int32_t blk = tile.block(i);
            const int buf = (i - i0) & 1;
            if (!kLate) read(i + 1, next);
            const MQ_LDS int8_t* from = lds + buf * kStage<DT> + at.lane * 16;
            v16f c[2];
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int x = 0; x < 16; ++x) c[j][x] = 0.0f;
#pragma unroll
            for (int u = 0; u < DT; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const v8h k = *reinterpret_cast<const MQ_LDS v8h*>(
                            from + (j * DT + u) * 2048 + h * 1024);
#pragma unroll
                        for (int e = 0; e < N; ++e) c[j] = mfma32(k, q[e][u][h], c[j]);
                    }
            if (!tile.full(p, blk) || __ballot(!(now.placed[0] && now.placed[1])) != 0) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    struct {
                        v16f& c;
                        __device__ float operator()(int i) const { return c[i]; }
                        __device__ void operator()(int i, float x) const { c[i] = x; }
                    } score{c[j]};
                    mask_scores(p, row.sees, blk * kBlk + 32 * j + 16 * at.hh, now.placed[j],
                                now.k[j], now.v[j], score);
                }
            }
            Weigh f[2];
            float most = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float x = c[j][0];
#pragma unroll
                for (int e = 1; e < 16; ++e) x = fmaxf(x, c[j][e]);
                most = fmaxf(most, f[j].top(qa, now.k[j], value_scale(now.v[j]), x));
            }
            uint32_t o;
            const uint32_t own = swap32(__builtin_bit_cast(uint32_t, most), o);
            most = fmaxf(__builtin_bit_cast(float, own), __builtin_bit_cast(float, o));
            if (__ballot(most - m > kLag) != 0) {  // (the sum could round up)
                most = fmaxf(most, m);
                const float down = exp2_fast(m - most);
                l *= down;
#pragma unroll
                for (int u = 0; u < DT; ++u) acc[u] *= down;
                m = most;
            }
            v8h w[2][2][N];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                f[j].b = f[j].lv + (kTop - m);
                if (__ballot(fabsf(m) >= kHuge) != 0) {
#pragma unroll
                    for (int x = 0; x < 16; ++x) c[j][x] = far_exponent(f[j], c[j][x], m);
                    f[j].a = 1.0f;
                    f[j].b = 0.0f;
                }
                float sum = 0.0f;
#pragma unroll
                for (int x = 0; x < 16; ++x) weigh(f[j], c[j][x], x & 7, w[j][x >> 3], sum);
                l = __builtin_fmaf(sum, f[j].iv, l);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int u = 0; u < DT; ++u) {
                        const v8h v = *reinterpret_cast<const MQ_LDS v8h*>(
                            from + ((2 + j) * DT + u) * 2048 + h * 1024);
#pragma unroll
                        for (int e = 0; e < N; ++e) acc[u] = mfma32(v, w[j][h][e], acc[u]);
                    }
            if (kLate) read(i + 1, next);
            put(buf ^ 1);
            now = next;
            __syncthreads();
        }
    }
    {
        uint32_t o;
        const uint32_t own = swap32(__builtin_bit_cast(uint32_t, l), o);
        l = __builtin_bit_cast(float, own) + __builtin_bit_cast(float, o);
    }
    if (!row.have) return;
    const int64_t part = (row.t * p.H + row.head) * p.splits + split;
    if (p.splits > 1 && at.hh == 0) {
        p.ml[2 * part] = m;
        p.ml[2 * part + 1] = l;
    }
    const float unit = out_unit(l);
    const int64_t out = out_at(p, row.t, row.head);
#pragma unroll
    for (int u = 0; u < DT; ++u)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int32_t d = 32 * u + 8 * x + 4 * at.hh;
            if (d >= p.kv.D) break;
            const v4f v = {acc[u][4 * x], acc[u][4 * x + 1], acc[u][4 * x + 2], acc[u][4 * x + 3]};
            if (p.splits > 1) *reinterpret_cast<v4f*>(p.sums + part * p.kv.D + d) = v;
            else store_four<N>(p, out, d, v * unit);
        }
}

// The parts of a call's rows: every sequence's tiles of 16 rows, its blocks split
// into parts of about the same size over all sequences.  Every work-group (and the
// join) works it out from the lengths for itself.
struct Plan {
    int32_t b;             // the work-group's sequence, or -1
    int32_t tile, part;    // its tile and part of it
    int32_t parts;         // of each of the sequence's tiles
    int32_t first;         // work-group of the tile's first part
    int32_t s0, s1, len;
};
// x: work-group, or (row >= 0) the work-group of that token row's first head of
// the group plus `head`.
__device__ inline Plan make_plan(const AttnArgs& p, int waves, int32_t x, int64_t token,
                                 int32_t head)
{
    const int lane = threadIdx.x & 63;
    int32_t s0[kPlanRegs], s1[kPlanRegs], len[kPlanRegs], tiles[kPlanRegs], n[kPlanRegs];
#pragma unroll
    for (int i = 0; i < kPlanRegs; ++i) {
        const int32_t b = min(lane + 64 * i, p.kv.B - 1);
        if (64 * i >= p.kv.B) {  // uniform
            s0[i] = s1[i] = len[i] = 0;
            continue;
        }
        s0[i] = p.kv.starts[b];
        s1[i] = p.kv.starts[b + 1];
        len[i] = p.kv.lens[b];
    }
    const int32_t list = (int32_t)min((p.kv.ld << p.kv.shift) / kBlk + 1, (int64_t)1 << 25);
    int64_t total = 0;
#pragma unroll
    for (int i = 0; i < kPlanRegs; ++i) {
        if (64 * i >= p.kv.B) break;
        const bool ok = lane + 64 * i < p.kv.B && s0[i] >= 0 && s1[i] <= (int32_t)p.T &&
                        s0[i] < s1[i];
        if (!ok) s1[i] = s0[i];
        const int32_t rows = ok ? s1[i] - s0[i] : 0;
        tiles[i] = (rows * p.grp + kRows - 1) / kRows;  // (T * grp <= 16 B on this path)
        // blocks up to the last token's, without those that a window hides from all
        const int32_t last = max(len[i], 0) - 1;
        int32_t end = last < 0 ? 0 : min(last / kBlk + 1, list);
        if (p.window > 0) {
            const int64_t seen = (int64_t)last - rows - p.window;  // hidden up to here
            const int32_t hide = (int32_t)(seen >> 6) - (int32_t)(((int64_t)p.sinks + kBlk - 1) >> 6);
            if (seen > 0) end -= max(min(hide, end), 0);
        }
        n[i] = max(end, 1);
        total += (int64_t)tiles[i] * n[i];
    }
    static_assert(kBlk == 64, "shifts");
    // blocks of a part: at least one per wave, whole rounds of the waves (waves: a
    // power of two)
    uint32_t per = waves;
    if (p.target > 0) {
        total = wave_sum(total);
        const double each = (double)total * (double)p.kv.G / (double)p.target;
        per = max(per, (uint32_t)min(each, 1073741824.0) + 1);
    }
    per = (per + waves - 1) & ~(uint32_t)(waves - 1);
    Plan w;
    w.b = -1;
    int32_t base = 0;
#pragma unroll
    for (int i = 0; i < kPlanRegs; ++i) {
        if (64 * i >= p.kv.B) break;
        int32_t parts = 1;
        if (p.target > 0)
            parts = (int32_t)min(max(((uint32_t)n[i] + per / 2) / per, 1u), (uint32_t)kMaxParts);
        const int32_t mine = tiles[i] * parts, after = wave_scan(mine);
        bool hit;
        if (token >= 0) hit = tiles[i] > 0 && token >= s0[i] && token < s1[i];
        else hit = x >= base + after - mine && x < base + after;
        const uint64_t at = __ballot(hit);
        if (at != 0 && w.b < 0) {
            const int l = 63 - __builtin_clzll(at);
            w.b = 64 * i + l;
            w.parts = __builtin_amdgcn_readlane(parts, l);
            w.s0 = __builtin_amdgcn_readlane(s0[i], l);
            w.s1 = __builtin_amdgcn_readlane(s1[i], l);
            w.len = __builtin_amdgcn_readlane(len[i], l);
            const int32_t before = base + __builtin_amdgcn_readlane(after - mine, l);
            if (token >= 0) {
                w.tile = (((int32_t)token - w.s0) * p.grp + head) / kRows;
                w.part = 0;
                // (starts that do not ascend: more work-groups than there are)
                if (before < 0 || (int64_t)before + (int64_t)(w.tile + 1) * w.parts > p.slots)
                    w.parts = 0;
            } else {
                w.tile = (int32_t)((uint32_t)(x - before) / (uint32_t)w.parts);
                w.part = x - before - w.tile * w.parts;
            }
            w.first = before + w.tile * w.parts;
        }
        base += __builtin_amdgcn_readlane(after, 63);
    }
    return w;
}

// grid (work-groups per head, G).  PLAN: parts by make_plan; else (more sequences)
// a work-group per tile of 16 rows.
template <int KS, int ND, int N, int W, bool PLAN>
__global__ __launch_bounds__(64 * W, KS <= 2 ? 2 : 1) void attn_blocks_rows_kernel(AttnArgs p)
{
    __shared__ __attribute__((aligned(16))) float lds[kJoinFloats<ND, W>];
    const int32_t g0 = blockIdx.y;
    Tile tile;
    int32_t i0 = 0, i1;
    PartAt part{true, 0};
    if constexpr (PLAN) {
        const Plan w = make_plan(p, W, (int32_t)blockIdx.x, -1, 0);
        if (w.b < 0) return;
        set_tile<kRows>(p, w.b, w.s0, w.s1, max(w.len, 0), (uint32_t)w.tile * kRows, tile);
        i1 = tile.n;
        if (w.parts > 1) {
            const int32_t per = (tile.n + w.parts - 1) / w.parts;
            i0 = per * w.part;
            i1 = min(i0 + per, tile.n);
            part.only = false;
            part.at = ((int64_t)g0 * p.slots + blockIdx.x) * kRows + (threadIdx.x & 15);
        }
    } else {
        if (!find_tile<kRows, kBlk>(p, blockIdx.x, tile)) return;
        i1 = tile.n;
    }
    const RowAt row(p, tile, tile.row0, g0);
    split_rows<KS, ND, N, W>(p, tile, g0, i0, i1, row, part, lds);
}

// One work-group per tile of rows, cache head and split; a sequence's last 16 rows
// or fewer are split among the waves.
template <int KS, int ND, int N>
__global__ __launch_bounds__(256, KS <= (N == 2 ? 1 : 2) ? 2 : 1) void attn_blocks_tile_kernel(
    AttnArgs p, int64_t tiles)
{
    constexpr int DT = ND / 2, kJoin = kJoinFloats<ND, kWaves> * 4;
    constexpr int kBytes = 2 * kStage<DT> > kJoin ? 2 * kStage<DT> : kJoin;
    __shared__ __attribute__((aligned(1024))) int8_t lds[kBytes];
    const Place w = place_of(p, blockIdx.x, tiles);
    const int32_t g0 = w.part % p.kv.G, split = w.part / p.kv.G;
    Tile tile;
    if (w.tile >= tiles || !find_tile<kTile, kBlk>(p, w.tile, tile)) return;
    int32_t i0, i1;
    split_range(p, tile, split, i0, i1);
    if (tile.rows - tile.row0 <= kRows) {
        const RowAt row(p, tile, tile.row0, g0);
        const PartAt part{p.splits == 1, (row.t * p.H + row.head) * p.splits + split};
        split_rows<KS, ND, N, kWaves>(p, tile, g0, i0, i1, row, part, reinterpret_cast<float*>(lds));
    } else {
        share_keys<DT, N>(p, tile, g0, i0, i1, split, (MQ_LDS int8_t*)lds);
    }
}

// Joins the parts of a row and head (PLAN: make_plan's, else the splits of tiles), a
// work-group per 64 channels: 16 lanes have four channels each of four parts at once,
// the four waves take turns; up to 128 parts' reads are under way together.
template <bool PLAN>
__global__ __launch_bounds__(256) void attn_blocks_join_kernel(AttnArgs p, int plan_waves)
{
    constexpr int kStep = PLAN ? kRows : 1;  // rows from a part's to the next one's
    __shared__ float f[kMaxParts];
    __shared__ __attribute__((aligned(16))) v4f sums[4][64];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x / p.H;
    const int32_t head = (int32_t)(blockIdx.x - t * p.H), D = p.kv.D;
    const int32_t g0 = head / p.grp, h = head - g0 * p.grp;
    int32_t parts;
    int64_t at;
    if constexpr (PLAN) {
        const Plan w = make_plan(p, plan_waves, 0, t, h);
        if (w.b < 0 || w.parts <= 1) return;  // rows of no sequence, or done
        parts = w.parts;
        at = ((int64_t)g0 * p.slots + w.first) * kRows + (((t - w.s0) * p.grp + h) & (kRows - 1));
    } else {
        if (t < p.kv.starts[0] || t >= p.kv.starts[p.kv.B]) return;
        parts = p.splits;
        at = (t * p.H + head) * parts;
    }
    const float* ml = p.ml + 2 * at;
    constexpr int kRegs = kMaxParts / 64;
    float m[kRegs], l[kRegs], most = kNone;
#pragma unroll
    for (int i = 0; i < kRegs; ++i) {
        const int s = lane + 64 * i;
        m[i] = s < parts ? ml[2 * kStep * s] : kNone;
        l[i] = s < parts ? ml[2 * kStep * s + 1] : 0.0f;
    }
    const int32_t which = 4 * wave + (lane >> 4), d = 64 * (int32_t)blockIdx.y + 4 * (lane & 15);
    const float* x = p.sums + at * D + min(d, D - 4);
    constexpr int U = 8;
    v4f v[U];
    auto load = [&](int32_t s0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t s = min(s0 + 16 * u + which, parts - 1);
            v[u] = *reinterpret_cast<const v4f*>(x + (int64_t)s * kStep * D);
        }
    };
    load(0);
#pragma unroll
    for (int i = 0; i < kRegs; ++i) most = fmaxf(most, m[i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor(most, o));
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kRegs; ++i) {
        const float e = exp2_fast(m[i] - most);
        if (wave == 0 && lane + 64 * i < parts) f[lane + 64 * i] = e;
        sum = __builtin_fmaf(e, l[i], sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    __syncthreads();
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int32_t s0 = 0; s0 < parts; s0 += 16 * U) {
        if (s0 > 0) load(s0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int32_t s = s0 + 16 * u + which;
            const float e = s < parts ? f[s] : 0.0f;
            if (s < parts)
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(e, v[u][c], acc[c]);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (threadIdx.x >= 16 || d >= D) return;
    acc = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 16; ++i) acc += sums[i >> 2][16 * (i & 3) + lane];
    store_four(p, out_at(p, t, head), d, acc * out_unit(sum));
}

// Joins the splits of tiles, a lane per four channels of a row and head.
__global__ __launch_bounds__(256) void attn_blocks_join_tiles_kernel(AttnArgs p)
{
    const uint32_t each = (uint32_t)p.kv.D / 4;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = i / each, t = row / p.H;
    const int32_t d = 4 * (int32_t)(i - row * each);
    if (row >= p.T * p.H || t < p.kv.starts[0] || t >= p.kv.starts[p.kv.B]) return;
    const float* ml = p.ml + row * p.splits * 2;
    const float* x = p.sums + row * p.splits * p.kv.D + d;
    float m = kNone, l = 0.0f;
    for (int s = 0; s < p.splits; ++s) m = fmaxf(m, ml[2 * s]);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < p.splits; ++s) {
        const float f = exp2_fast(ml[2 * s] - m);
        l = __builtin_fmaf(f, ml[2 * s + 1], l);
        const v4f v = *reinterpret_cast<const v4f*>(x + (int64_t)s * p.kv.D);
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[c] = __builtin_fmaf(f, v[c], acc[c]);
    }
    store_four(p, out_at(p, t, (int32_t)(row - t * p.H)), d, acc * out_unit(l));
}

// Whether the sequences have more rows than a set, on average.  (One kernel for all: 200
// sequences with a token over 1000 keys and one of 500 over 16000, 32 heads of 128 on 8,
// take 527 us in one call, whose 125 tiles of 16 rows read the chunk's keys each, 260 in
// two.)
bool tiled(int64_t T, int64_t B, int32_t grp) { return T * grp > B * kRows; }

// Work-groups that the chip holds at once (of rows: one of eight waves per CU, or
// of four with the registers of a wave per SIMD; of tiles: two per CU, or one).
constexpr int64_t kCUs = 256;

// How the keys are split: `splits` of every tile, or planned parts.
struct Split {
    int64_t splits = 1, target = 0, slots = 0, bytes = 0;
    int waves = 0;  // of a work-group of rows
};
Split choose_split(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D, int64_t max_len,
                   int64_t ws_bytes)
{
    Split c;
    const int32_t grp = H / G;
    const int64_t blocks = (max_len + kBlk - 1) / kBlk, row = (D + 2) * 4;
    ws_bytes = std::min<int64_t>(ws_bytes, MQ_ATTN_MAX_WORKSPACE);
    if (tiled(T, B, grp)) {
        // at least a block per wave in each
        // (tiles as of sequences with as many rows each; work-groups of one round: 240 tokens
        // of two sequences over 15000 keys, 8 heads of 256 on one, in 272 work-groups 119 us,
        // in 256 72)
        const int64_t seqs = std::min(B, T);
        const int64_t groups = seqs * ((T * grp + seqs * kTile - 1) / (seqs * kTile)) * G;
        int64_t s = (D > 128 ? kCUs : 2 * kCUs) / groups;
        s = std::min(s, (blocks + kWaves - 1) / kWaves);
        s = std::min<int64_t>(s, ws_bytes / (T * H * row));
        c.splits = std::max<int64_t>(1, std::min<int64_t>(s, kMaxParts));
        c.bytes = c.splits > 1 ? c.splits * T * H * row : 0;
        return c;
    }
    const int64_t tiles = row_tiles(T, B, grp, kRows);
    c.slots = tiles;
    // eight waves on a CU: one work-group of a few tiles', two of many's (one token over
    // 1531 keys, 32 heads of 64 on 4: 8.6 us, 10.7 with four waves; 64 sequences of 1000,
    // 32 heads of 128 on 8: 24.9 with four, 31.8 with eight); above 128 channels their
    // registers leave one wave per SIMD
    c.waves = D > 128 || std::min(tiles, std::max<int64_t>(B, T * grp / kRows)) * G > kCUs ? 4 : 8;
    // Up to four blocks per wave are one part's, whose launch needs no join (1531 keys: 8.6
    // us, 10.7 in parts; 3000 keys: 10.9 in parts, 12.5 in one; 8000: 11.0 and 25.6), eight
    // where the sequences alone fill the chip (200 of 1000 keys: 89 us, 120 in parts).
    if (B > kPlanned || blocks <= (std::min(B, T) * G >= kCUs ? 8 : 4) * c.waves) return c;
    const int64_t target = D > 128 || c.waves == 8 ? kCUs : 2 * kCUs;
    const int64_t slots = tiles + (target + G - 1) / G;
    if (slots * G * kRows * row > ws_bytes) return c;
    c.target = target;
    c.slots = slots;
    c.bytes = slots * G * kRows * row;
    return c;
}

template <int ND, int N, int W>
hipError_t launch_rows(const AttnArgs& p, hipStream_t s)
{
    constexpr int KS = (ND + 3) / 4;
    const dim3 grid((unsigned)p.slots, (unsigned)p.kv.G);
    if (p.kv.B <= kPlanned)
        attn_blocks_rows_kernel<KS, ND, N, W, true><<<grid, 64 * W, 0, s>>>(p);
    else
        attn_blocks_rows_kernel<KS, ND, N, W, false><<<grid, 64 * W, 0, s>>>(p);
    return hipGetLastError();
}

template <int ND, int N>
hipError_t launch_main(const AttnArgs& p, const Split& c, hipStream_t s)
{
    constexpr int KS = (ND + 3) / 4;
    if (c.waves > 0) {
        // (kMaxBlocks is of 256 threads)
        if (c.slots * p.kv.G * (c.waves / 4) >= kMaxBlocks) return hipErrorInvalidConfiguration;
        if constexpr (ND <= 8)
            if (c.waves == 8) return launch_rows<ND, N, 8>(p, s);
        return launch_rows<ND, N, 4>(p, s);
    }
    const int64_t parts = (int64_t)p.kv.G * p.splits;
    const int64_t tiles = row_tiles(p.T, p.kv.B, p.grp, kTile);
    // (see place_of)
    const int64_t n = parts % 8 != 0 && 8 % parts == 0
                          ? 8 * ((tiles + 8 / parts - 1) / (8 / parts))
                          : tiles * parts;
    if (n >= kMaxBlocks) return hipErrorInvalidConfiguration;
    attn_blocks_tile_kernel<KS, ND, N><<<(unsigned)n, 256, 0, s>>>(p, tiles);
    return hipGetLastError();
}

template <int ND>
hipError_t launch_terms(const AttnArgs& p, const Split& c, hipStream_t s)
{
    return p.type == MQ_F32 ? launch_main<ND, 2>(p, c, s) : launch_main<ND, 1>(p, c, s);
}

}  // namespace

int64_t attn_blocks_workspace(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D,
                              int64_t max_len)
{
    if (T == 0 || B == 0) return 0;
    return choose_split(T, B, H, G, D, max_len, MQ_ATTN_MAX_WORKSPACE).bytes;
}

hipError_t launch_attn_blocks(const BlockCache& c, const void* q, int64_t ldq, int32_t type,
                              int64_t T, int32_t H, float logit_scale, int64_t window,
                              int64_t sinks, void* y, int64_t ldy, int64_t max_len, void* ws,
                              int64_t ws_bytes, hipStream_t s)
{
    AttnArgs p;
    p.kv = c.kv;
    if (c.kv.pages == 0) p.kv.ld = 0;  // no place: no block is looked at
    p.k_scale = c.k_scale;
    p.v_scale = c.v_scale;
    p.bshift = c.bshift;
    p.type = type;
    p.q = q;
    p.y = y;
    p.ldq = ldq;
    p.ldy = ldy;
    p.T = T;
    p.H = H;
    p.grp = H / c.kv.G;
    p.tau = (float)((double)logit_scale * 1.4426950408889634);  // log2(e)
    // positions are below 2^31: a window of as many hides nothing
    p.window = window < 0x7FFFFFFF ? (int32_t)window : 0;
    p.sinks = p.window > 0 ? (int32_t)std::min<int64_t>(sinks, 0x7FFFFFFF) : 0;
    p.page_bytes = (c.kv.G * c.kv.D) << c.kv.shift;
    const int e = type_bytes(type);
    p.vec_q = (uintptr_t)q % 16 == 0 && ldq * e % 16 == 0;
    p.vec_y = (uintptr_t)y % (4 * e) == 0 && ldy % 4 == 0;
    // the blocks that a row of a windowed call walks over
    if (p.window > 0 && window < max_len)
        max_len = std::min(max_len, window + std::min<int64_t>(p.sinks, max_len) + 2 * kBlk);
    const Split split = choose_split(T, c.kv.B, H, c.kv.G, c.kv.D, max_len, ws ? ws_bytes : 0);
    if (split.slots > 0x7FFFFFFF) return hipErrorInvalidConfiguration;
    p.splits = (int32_t)split.splits;
    p.target = (int32_t)split.target;
    p.slots = (int32_t)split.slots;
    p.sums = static_cast<float*>(ws);
    p.ml = p.sums + split.bytes / ((c.kv.D + 2) * 4) * c.kv.D;
    hipError_t err;
    switch ((c.kv.D + 31) / 32) {
    case 1: err = launch_terms<2>(p, split, s); break;
    case 2: err = launch_terms<4>(p, split, s); break;
    case 3: err = launch_terms<6>(p, split, s); break;
    case 4: err = launch_terms<8>(p, split, s); break;
    case 5: err = launch_terms<10>(p, split, s); break;
    case 6: err = launch_terms<12>(p, split, s); break;
    case 7: err = launch_terms<14>(p, split, s); break;
    default: err = launch_terms<16>(p, split, s); break;
    }
    if (err != hipSuccess || split.bytes == 0) return err;
    // (T * H is far below the number of work-groups of a launch: two parts of every row
    // fit the workspace)
    const dim3 grid((unsigned)(T * H), (unsigned)((c.kv.D + 63) / 64));
    if (split.target > 0) {
        attn_blocks_join_kernel<true><<<grid, 256, 0, s>>>(p, split.waves);
    } else if (T * H * (c.kv.D / 4) <= kCUs * 256) {
        // (a lane's splits in turn where the rows fill the chip: 128 rows of 64 splits of 256
        // channels 4.7 us, 25 in turn; 1920 of 16 splits 10.8 in turn, 17.6)
        attn_blocks_join_kernel<false><<<grid, 256, 0, s>>>(p, 0);
    } else {
        const int64_t n = (T * H * (c.kv.D / 4) + 255) / 256;
        attn_blocks_join_tiles_kernel<<<(unsigned)n, 256, 0, s>>>(p);
    }
    return hipGetLastError();
}

}  // namespace mq
