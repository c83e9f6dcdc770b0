// Attention of new tokens over the cache with block scales, in one pass with a
// running maximum, scores and weights in registers throughout.
//
// A wave holds 16 rows (a row: one token's query head; the H / G heads that
// share a cache head lie next to each other) per set and walks over blocks of 64
// key positions.  Both products run on the fp16 matrix instructions with fp32
// sums: codes are exact in fp16, the queries of a row are scaled by a power of
// two to below 2^15, which leaves bf16 and fp16 queries exact, fp32 ones as the
// sum of two fp16 numbers (22 bits).  Scores come out transposed,
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
// outputs to the sum of two; statistics and outputs are fp32.
#include <algorithm>
#include <cmath>

#include "kvblocks.h"
#include "kvwalk.h"
#include "mq_internal.h"
#include "tokens.h"

#define MQ_LDS __attribute__((address_space(3)))
#define MQ_GLOBAL __attribute__((address_space(1)))

namespace mq {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int kBlk = 64;                  // key positions per step
constexpr int kRows = 16;                 // rows per set
constexpr int kWaves = 4;                 // waves per work-group
// sets per wave where the waves share keys (fp32 rows of more than 192 channels
// leave registers for one)
template <int KS, int N>
constexpr int kSets = KS == 4 && N == 2 ? 1 : 2;
template <int KS, int N>
constexpr int kTile = kRows * kSets<KS, N> * kWaves;
constexpr int kMaxSplits = 256;
constexpr float kNone = -1e30f;           // running maximum of a row that has seen nothing
constexpr float kTop = 8.0f, kLag = 7.0f; // weights up to 2^(kTop + kLag)
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
    int32_t splits;
    float* ml;             // [T * H][splits][2]: maximum and weight sum of a part
    float* sums;           // [T * H][splits][D]
};

__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline v4f mfma(v8h a, v8h b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// 16 codes as fp16, exact: the byte c + 128 in the low bits of 1024 is 1152 + c.
__device__ inline void to_half(const v4i& x, v8h (&h)[2])
{
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    const v2h off = {(_Float16)-1152.0f, (_Float16)-1152.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = (uint32_t)x[i] ^ 0x80808080u;
        const v2h lo = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) + off;
        const v2h hi = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) + off;
        h[i >> 1][4 * (i & 1)] = lo[0];
        h[i >> 1][4 * (i & 1) + 1] = lo[1];
        h[i >> 1][4 * (i & 1) + 2] = hi[0];
        h[i >> 1][4 * (i & 1) + 3] = hi[1];
    }
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

// A set of 16 rows: KS steps of 64 channels, ND tiles of 16 output channels, N
// fp16 terms of queries and of weights.
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

template <int TYPE>
__device__ inline void load16(const AttnArgs& p, int64_t i, float (&x)[16])
{
    constexpr int E = TYPE == MQ_F32 ? 4 : 2;
    if (p.vec_q) {
        Raw<TYPE, 16> r;
        r.load(static_cast<const int8_t*>(p.q) + i * E);
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = r[j];
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = load_elem<TYPE>(p.q, i + j);
    }
}

// N == 2: fp32 queries.  Channels past the head and rows past the tile are 0.
template <int KS, int ND, int N>
__device__ inline void load_queries(const AttnArgs& p, const RowAt& row, Rows<KS, ND, N>& st)
{
    const int g = (threadIdx.x & 63) >> 4;
    const int64_t at = row.t * p.ldq + (int64_t)row.head * p.kv.D;
    float x[KS][16];
    float most = 0.0f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
        const int d = 64 * s + 16 * g;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[s][j] = 0.0f;
        if (row.have && d < p.kv.D) {
            if constexpr (N == 2) load16<MQ_F32>(p, at + d, x[s]);
            else if (p.type == MQ_BF16) load16<MQ_BF16>(p, at + d, x[s]);
            else load16<MQ_F16>(p, at + d, x[s]);
        }
#pragma unroll
        for (int j = 0; j < 16; ++j) most = fmaxf(most, fabsf(x[s][j]));
    }
    most = row_max(most);
    // 2^e <= most < 2^(e + 1); the row times 2^(14 - e), the products by its inverse
    const uint32_t e = min(max(abs_bits(most) >> 23, 27u), 254u);
    const float up = __builtin_bit_cast(float, (268u - e) << 23);
    st.a = p.tau * __builtin_bit_cast(float, (e - 14u) << 23);
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float v = x[s][j] * up;
            const _Float16 h = (_Float16)v;
            st.q[0][s][j >> 3][j & 7] = h;
            if constexpr (N == 2) st.q[1][s][j >> 3][j & 7] = (_Float16)(v - (float)h);
        }
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
    int64_t scale;
    bool placed;  // the value group
    __device__ Addr(const AttnArgs& p, const Tile& t, int32_t g0, int32_t blk, const Pages& pg)
    {
        const Spot s;
        const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
        const int32_t mask = (1 << p.kv.shift) - 1;
        const int32_t kp = is_page(p, t, blk, s.key, pg.key) ? pg.key : 0;
        placed = is_page(p, t, blk, s.value, pg.value);
        const int32_t vp = placed ? pg.value : 0;
        const int32_t ks = (blk * kBlk + 16 * s.key) & mask, vs = (blk * kBlk + 16 * s.value) & mask;
        const int64_t head = (int64_t)g0 << p.kv.shift;
        k = (const MQ_GLOBAL int8_t*)p.kv.k +
            ((uint64_t)(uint32_t)kp * (uint32_t)p.page_bytes +
             (uint64_t)((head + ks + (r & 3)) * p.kv.D + 16 * g));
        v = (const MQ_GLOBAL int8_t*)p.kv.v +
            ((uint64_t)(uint32_t)vp * (uint32_t)p.page_bytes +
             (uint64_t)((head + vs) * p.kv.D + 16 * r));
        scale = (((int64_t)vp * p.kv.G + g0) << (p.kv.shift - p.bshift)) + (vs >> p.bshift);
    }
};

// Channels past the head dimension: the scores read the head's first ones again
// (the queries are 0 there), the outputs of such a tile are dropped.
__device__ inline int32_t key_chunk(const AttnArgs& p, int s)
{
    const int32_t c = 16 * ((threadIdx.x & 63) >> 4);
    return 64 * s + c < p.kv.D ? 64 * s : -c;
}
__device__ inline int32_t value_tile(const AttnArgs& p, int dt)
{
    return 16 * dt < p.kv.D ? 256 * dt : 0;
}

// One block for the wave's sets.  key(j, s), value(dt): fragments; read():
// called once the keys have been used; ks, vs: the lane's scales, placed: whether
// its group has a place; full: every row sees every position.
template <int KS, int ND, int N, int NR, class Key, class Value, class Read>
__device__ inline void attend_block(const AttnArgs& p, Rows<KS, ND, N> (&st)[NR],
                                    const Sees (&sees)[NR], int32_t blk, bool full, bool placed,
                                    float ks, float vs, Key key, Value value, Read read)
{
    const int g = (threadIdx.x & 63) >> 4;
    // scores of keys 16 g + 4 j + i
    v4f c[NR][4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            v8h k[2];
            to_half(key(j, s), k);
#pragma unroll
            for (int n = 0; n < NR; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < N; ++e)
                        c[n][j] = mfma(k[h], st[n].q[e][s][h],
                                       s + h + e ? c[n][j] : v4f{0.0f, 0.0f, 0.0f, 0.0f});
        }
    read();
    const bool mask = !full || __ballot(!placed) != 0;
    v8h w[NR][N][2];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        uint32_t seen = 0xffff;
        float kn = ks, vn = fmaxf(vs, 0x1p-67f);
        if (mask) {
            const int32_t first = blk * kBlk + 16 * g;
            // of the 16 keys from `first` on those below x, as bits
            auto below = [&](int32_t x) { return (1u << max(min(x - first, 16), 0)) - 1; };
            seen = below(sees[n].hi + 1) & (~below(sees[n].lo + 1) | below(p.sinks));
            if (!placed) seen = 0;
            if (seen == 0) kn = vn = 1.0f;  // (the scales there may be anything)
        }
        const float a = st[n].a * kn, lv = __builtin_amdgcn_logf(vn);
        float x[16], m;
        if (mask) {
            m = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] = __builtin_fmaf(c[n][i >> 2][i & 3], a, lv);
                x[i] = (seen >> i) & 1 ? x[i] : -__builtin_inff();
                m = fmaxf(m, x[i]);
            }
        } else {
            m = c[n][0][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) m = fmaxf(m, c[n][i >> 2][i & 3]);
            m = __builtin_fmaf(m, a, lv);
        }
        m = row_max(m);
        if (__ballot(m > st[n].m + kLag) != 0) {
            m = fmaxf(m, st[n].m);
            const float f = exp2_fast(st[n].m - m);
            st[n].l *= f;
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) st[n].acc[dt] *= f;
            st[n].m = m;
        }
        const float b = kTop - st[n].m;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            x[i] = exp2_fast(mask ? x[i] + b : __builtin_fmaf(c[n][i >> 2][i & 3], a, lv + b));
            sum += x[i];
        }
        st[n].l = __builtin_fmaf(sum, exp2_fast(-lv), st[n].l);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const _Float16 h = (_Float16)x[i];
            w[n][0][i >> 3][i & 7] = h;
            if constexpr (N == 2) w[n][1][i >> 3][i & 7] = (_Float16)(x[i] - (float)h);
        }
    }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        v8h v[2];
        to_half(value(dt), v);
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int e = 0; e < N; ++e) st[n].acc[dt] = mfma(v[h], w[n][e][h], st[n].acc[dt]);
    }
}

// 1 / l; 0 for a row that sees nothing.
__device__ inline float out_unit(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

__device__ inline void store_one(const AttnArgs& p, int64_t t, int32_t head, int32_t d, float v)
{
    const int64_t at = t * p.ldy + (int64_t)head * p.kv.D + d;
    if (p.type == MQ_F32) store_elem<MQ_F32>(p.y, at, v);
    else if (p.type == MQ_BF16) store_elem<MQ_BF16>(p.y, at, v);
    else store_elem<MQ_F16>(p.y, at, v);
}
__device__ inline void store_four(const AttnArgs& p, int64_t t, int32_t head, int32_t d, v4f v)
{
    const int64_t at = t * p.ldy + (int64_t)head * p.kv.D + d;
    if (!p.vec_y) {
#pragma unroll
        for (int i = 0; i < 4; ++i) store_one(p, t, head, d + i, v[i]);
    } else if (p.type == MQ_F32) {
        *reinterpret_cast<v4f*>(static_cast<float*>(p.y) + at) = v;
    } else {
        const uint2 h = p.type == MQ_BF16
                            ? make_uint2(pack2<MQ_BF16>(v[0], v[1]), pack2<MQ_BF16>(v[2], v[3]))
                            : make_uint2(pack2<MQ_F16>(v[0], v[1]), pack2<MQ_F16>(v[2], v[3]));
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p.y) + at) = h;
    }
}

// Four waves share 16 rows and take every fourth block of [i0, i1), straight from
// the cache; their states are joined through LDS.
template <int ND>
constexpr int kJoinFloats = kWaves * (4 * ND * 64 + 2 * kRows);
template <int KS, int ND, int N>
__device__ inline void split_rows(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, int split, float* lds)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const RowAt row(p, tile, tile.row0, g0);
    const Sees sees[1] = {row.sees};
    Rows<KS, ND, N> st[1];
    st[0].clear();
    int32_t i = i0 + wave;
    if (i < i1) {
        Pages pg = load_pages(p, tile, tile.block(i));
        load_queries(p, row, st[0]);
        v4i kf[4][KS];
        float ks, vs;
        Addr at(p, tile, g0, tile.block(i), pg);
        auto read_keys = [&]() {
            ks = p.k_scale[at.scale];
            vs = p.v_scale[at.scale];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    kf[j][s] = *reinterpret_cast<const MQ_GLOBAL v4i*>(
                        at.k + (4 * j * p.kv.D + key_chunk(p, s)));
        };
        read_keys();
        pg = load_pages(p, tile, tile.block(min(i + kWaves, i1 - 1)));
        for (; i < i1; i += kWaves) {
            const int32_t blk = tile.block(i);
            v4i vf[ND];
#pragma unroll
            for (int dt = 0; dt < ND; ++dt)
                vf[dt] = *reinterpret_cast<const MQ_GLOBAL v4i*>(at.v + value_tile(p, dt));
            const float ks0 = ks, vs0 = vs;
            const bool placed = at.placed;
            attend_block<KS, ND, N, 1>(
                p, st, sees, blk, tile.full(p, blk), placed, ks0, vs0,
                [&](int j, int s) { return kf[j][s]; }, [&](int dt) { return vf[dt]; },
                [&]() {
                    const int32_t next = tile.block(min(i + kWaves, i1 - 1));
                    at = Addr(p, tile, g0, next, pg);
                    read_keys();
                    pg = load_pages(p, tile, tile.block(min(i + 2 * kWaves, i1 - 1)));
                });
        }
    }
    float* lm = lds + kWaves * 4 * ND * 64;  // [wave][row]
    float* ll = lm + kWaves * kRows;
    const float l = row_sum(st[0].l);
    if (g == 0) {
        lm[wave * kRows + r] = st[0].m;
        ll[wave * kRows + r] = l;
    }
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) lds[((wave * ND + dt) * 4 + e) * 64 + lane] = st[0].acc[dt][e];
    __syncthreads();
    float m = kNone;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, lm[w * kRows + r]);
    float f[kWaves], sum = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        f[w] = exp2_fast(lm[w * kRows + r] - m);
        sum = __builtin_fmaf(f[w], ll[w * kRows + r], sum);
    }
    if (!row.have) return;
    const int64_t part = (row.t * p.H + row.head) * p.splits + split;
    if (p.splits > 1 && wave == 0 && g == 0) {
        p.ml[2 * part] = m;
        p.ml[2 * part + 1] = sum;
    }
    const float unit = out_unit(sum);
#pragma unroll
    for (int dt = wave; dt < ND; dt += kWaves) {
        const int32_t d = 16 * dt + 4 * g;
        if (16 * dt >= p.kv.D) break;
        v4f v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = __builtin_fmaf(f[w], lds[((w * ND + dt) * 4 + e) * 64 + lane], v[e]);
        if (p.splits > 1) *reinterpret_cast<v4f*>(p.sums + part * p.kv.D + d) = v;
        else store_four(p, row.t, row.head, d, v * unit);
    }
}

// The wave's own copies into LDS have landed (they count as vector memory).
__device__ inline void wait_staged()
{
    __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));  // vmcnt(0), the others left alone
}

// Every wave has sets of its own; all walk over blocks [i0, i1), staged in LDS by
// the four together in the order of the lanes (keys (j, s), then values: 1 KB
// each), the next block on its way during this one.
template <int KS, int ND>
constexpr int kStage = (4 * KS + ND) * 1024;
template <int KS, int ND, int N>
__device__ inline void share_keys(const AttnArgs& p, const Tile& tile, int32_t g0, int32_t i0,
                                  int32_t i1, int split, MQ_LDS int8_t* lds)
{
    const int lane = threadIdx.x & 63, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    constexpr int NR = kSets<KS, N>;
    RowAt row[NR];
    Sees sees[NR];
    Rows<KS, ND, N> st[NR];
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        row[n] = RowAt(p, tile, tile.row0 + kRows * (NR * wave + n), g0);
        sees[n] = row[n].sees;
        st[n].clear();
    }
    if (i0 < i1) {
        Pages pg = load_pages(p, tile, tile.block(i0));
        float ks = 0.0f, vs = 0.0f;
        bool placed = false;
        // the wave's share: key tile j = wave, every fourth value tile
        auto stage = [&](int32_t blk, MQ_LDS int8_t* to) {
            const Addr at(p, tile, g0, blk, pg);
            ks = p.k_scale[at.scale];
            vs = p.v_scale[at.scale];
            placed = at.placed;
#pragma unroll
            for (int s = 0; s < KS; ++s)
                __builtin_amdgcn_global_load_lds(
                    (const MQ_GLOBAL void*)(at.k + (4 * wave * p.kv.D + key_chunk(p, s))),
                    (MQ_LDS void*)(to + (wave * KS + s) * 1024), 16, 0, 0);
#pragma unroll
            for (int i = 0; i < (ND + 3) / 4; ++i) {
                const int dt = 4 * i + wave;
                if (dt < ND)
                    __builtin_amdgcn_global_load_lds(
                        (const MQ_GLOBAL void*)(at.v + value_tile(p, dt)),
                        (MQ_LDS void*)(to + (4 * KS + dt) * 1024), 16, 0, 0);
            }
        };
        stage(tile.block(i0), lds);
        pg = load_pages(p, tile, tile.block(min(i0 + 1, i1 - 1)));
#pragma unroll
        for (int n = 0; n < NR; ++n) load_queries(p, row[n], st[n]);
        wait_staged();
        __syncthreads();
        for (int32_t i = i0; i < i1; ++i) {
            const int32_t blk = tile.block(i);
            const int buf = (i - i0) & 1;
            const float ks0 = ks, vs0 = vs;
            const bool placed0 = placed;
            if (i + 1 < i1) {
                stage(tile.block(i + 1), lds + (buf ^ 1) * kStage<KS, ND>);
                pg = load_pages(p, tile, tile.block(min(i + 2, i1 - 1)));
            }
            const MQ_LDS int8_t* at = lds + buf * kStage<KS, ND> + lane * 16;
            attend_block<KS, ND, N, NR>(
                p, st, sees, blk, tile.full(p, blk), placed0, ks0, vs0,
                [&](int j, int s) {
                    return *reinterpret_cast<const MQ_LDS v4i*>(at + (j * KS + s) * 1024);
                },
                [&](int dt) {
                    return *reinterpret_cast<const MQ_LDS v4i*>(at + (4 * KS + dt) * 1024);
                },
                []() {});
            wait_staged();
            __syncthreads();
        }
    }
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        const float l = row_sum(st[n].l);
        if (!row[n].have) continue;
        const int64_t part = (row[n].t * p.H + row[n].head) * p.splits + split;
        if (p.splits > 1 && g == 0) {
            p.ml[2 * part] = st[n].m;
            p.ml[2 * part + 1] = l;
        }
        const float unit = out_unit(l);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
            if (16 * dt >= p.kv.D) break;
            const int32_t d = 16 * dt + 4 * g;
            if (p.splits > 1) *reinterpret_cast<v4f*>(p.sums + part * p.kv.D + d) = st[n].acc[dt];
            else store_four(p, row[n].t, row[n].head, d, st[n].acc[dt] * unit);
        }
    }
}

// grid (tiles of 16 rows, G, splits)
template <int KS, int ND, int N>
__global__ __launch_bounds__(256, KS <= 2 ? 2 : 1) void attn_blocks_split_kernel(AttnArgs p)
{
    __shared__ __attribute__((aligned(16))) float lds[kJoinFloats<ND>];
    Tile tile;
    if (!find_tile<kRows, kBlk>(p, blockIdx.x, tile)) return;
    int32_t i0, i1;
    split_range(p, tile, blockIdx.z, i0, i1);
    split_rows<KS, ND, N>(p, tile, blockIdx.y, i0, i1, blockIdx.z, lds);
}

// One work-group per tile of rows, cache head and split; a sequence's last 16 rows
// or fewer are split among the waves.
template <int KS, int ND, int N>
__global__ __launch_bounds__(256, KS <= 2 ? 2 : 1) void attn_blocks_tile_kernel(AttnArgs p,
                                                                                int64_t tiles)
{
    constexpr int kBytes = 2 * kStage<KS, ND> > kJoinFloats<ND> * 4 ? 2 * kStage<KS, ND>
                                                                    : kJoinFloats<ND> * 4;
    __shared__ __attribute__((aligned(1024))) int8_t lds[kBytes];
    const Place w = place_of(p, blockIdx.x, tiles);
    const int32_t g0 = w.part % p.kv.G, split = w.part / p.kv.G;
    Tile tile;
    if (w.tile >= tiles || !find_tile<kTile<KS, N>, kBlk>(p, w.tile, tile)) return;
    int32_t i0, i1;
    split_range(p, tile, split, i0, i1);
    if (tile.rows - tile.row0 <= kRows)
        split_rows<KS, ND, N>(p, tile, g0, i0, i1, split, reinterpret_cast<float*>(lds));
    else
        share_keys<KS, ND, N>(p, tile, g0, i0, i1, split, (MQ_LDS int8_t*)lds);
}

// Joins the splits: a wave per row and 64 channels.
__global__ __launch_bounds__(256) void attn_blocks_join_kernel(AttnArgs p)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= p.T * p.H) return;
    const int64_t t = row / p.H;
    if (t < p.kv.starts[0] || t >= p.kv.starts[p.kv.B]) return;  // rows of no sequence
    const int32_t d = blockIdx.y * 64 + lane;
    const bool have = d < p.kv.D;
    const float* ml = p.ml + row * p.splits * 2;
    const float* x = p.sums + row * p.splits * p.kv.D + (have ? d : 0);
    float m = kNone;
    for (int s = lane; s < p.splits; s += 64) m = fmaxf(m, ml[2 * s]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
    float l = 0.0f, acc = 0.0f;
    for (int s = 0; s < p.splits; ++s) {
        const float f = exp2_fast(ml[2 * s] - m);
        l = __builtin_fmaf(f, ml[2 * s + 1], l);
        acc = __builtin_fmaf(f, x[(int64_t)s * p.kv.D], acc);
    }
    if (have) store_one(p, t, (int32_t)(row % p.H), d, acc * out_unit(l));
}

// Whether the sequences have more rows than a set, on average.
bool tiled(int64_t T, int64_t B, int32_t grp) { return T * grp > B * kRows; }

// Parts the keys of every tile are split into: as many work-groups as the chip
// holds at once, at least a block per wave in each.
int64_t split_count(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D, int64_t max_len)
{
    const int32_t grp = H / G;
    const int R = tiled(T, B, grp) ? kTile<1, 1> : kRows;
    const int64_t groups = std::max(T * grp / R, std::min(B, T)) * G;
    int64_t s = (D > 128 ? 256 : 512) / std::max<int64_t>(groups, 1);
    const int64_t blocks = (max_len + kBlk - 1) / kBlk;
    s = std::min(s, (blocks + kWaves - 1) / kWaves);
    s = std::min<int64_t>(s, MQ_ATTN_MAX_WORKSPACE / (T * H * (D + 2) * 4));
    return std::max<int64_t>(1, std::min<int64_t>(s, kMaxSplits));
}

template <int ND, int N>
hipError_t launch_main(const AttnArgs& p, int64_t B, hipStream_t s)
{
    constexpr int KS = (ND + 3) / 4;
    const int64_t parts = (int64_t)p.kv.G * p.splits;
    if (tiled(p.T, B, p.grp)) {
        const int64_t tiles = row_tiles(p.T, B, p.grp, kTile<KS, N>);
        // (see place_of)
        const int64_t n = parts % 8 != 0 && 8 % parts == 0
                              ? 8 * ((tiles + 8 / parts - 1) / (8 / parts))
                              : tiles * parts;
        if (n >= kMaxBlocks) return hipErrorInvalidConfiguration;
        attn_blocks_tile_kernel<KS, ND, N><<<(unsigned)n, 256, 0, s>>>(p, tiles);
        return hipGetLastError();
    }
    const int64_t n = row_tiles(p.T, B, p.grp, kRows);
    if (n >= kMaxBlocks) return hipErrorInvalidConfiguration;
    const dim3 grid((unsigned)n, (unsigned)p.kv.G, (unsigned)p.splits);
    attn_blocks_split_kernel<KS, ND, N><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <int ND>
hipError_t launch_terms(const AttnArgs& p, int64_t B, hipStream_t s)
{
    return p.type == MQ_F32 ? launch_main<ND, 2>(p, B, s) : launch_main<ND, 1>(p, B, s);
}

}  // namespace

int64_t attn_blocks_workspace(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D,
                              int64_t max_len)
{
    if (T == 0 || B == 0) return 0;
    const int64_t s = split_count(T, B, H, G, D, max_len);
    return s > 1 ? s * T * H * (D + 2) * 4 : 0;
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
    int64_t splits = split_count(T, c.kv.B, H, c.kv.G, c.kv.D, max_len);
    const int64_t one = T * H * (c.kv.D + 2) * 4;
    splits = ws ? std::min(splits, std::max<int64_t>(ws_bytes / one, 1)) : 1;
    p.splits = (int32_t)splits;
    p.sums = static_cast<float*>(ws);
    p.ml = p.sums + T * H * splits * c.kv.D;
    hipError_t err;
    switch ((c.kv.D + 31) / 32) {
    case 1: err = launch_terms<2>(p, c.kv.B, s); break;
    case 2: err = launch_terms<4>(p, c.kv.B, s); break;
    case 3: err = launch_terms<6>(p, c.kv.B, s); break;
    case 4: err = launch_terms<8>(p, c.kv.B, s); break;
    case 5: err = launch_terms<10>(p, c.kv.B, s); break;
    case 6: err = launch_terms<12>(p, c.kv.B, s); break;
    case 7: err = launch_terms<14>(p, c.kv.B, s); break;
    default: err = launch_terms<16>(p, c.kv.B, s); break;
    }
    if (err != hipSuccess || splits == 1) return err;
    attn_blocks_join_kernel<<<dim3((unsigned)((T * H + 3) / 4), (unsigned)((c.kv.D + 63) / 64)),
                              256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mq
