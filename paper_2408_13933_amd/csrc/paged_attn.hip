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
#include <algorithm>
#include <cmath>

#include "codes.h"
#include "kvcache.h"
#include "mq_internal.h"
#include "requant.h"

namespace mq {
namespace {

constexpr int kBlk = MQ_ATTN_BLOCK;
constexpr int kRows = 16;   // rows per wave
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
    int64_t window, sinks;
    int32_t vec;          // 16-byte aligned query rows
    int32_t splits;
    double* part;         // [splits][T * H][D + 2] when splits > 1
};

constexpr double kLog2One = 0x1.dfa34e1177c23p+3;  // log2(MQ_ATTN_ONE)

// factor between two block maxima, 2^(-tau (hi - lo)), hi >= lo
__device__ inline double factor(const AttnArgs& p, int32_t hi, int32_t lo)
{
    return exp2_poly(fmax(-p.tau * ((double)hi - (double)lo), -1100.0));
}

__device__ inline v4i mfma(v4i a, v4i b, v4i c)
{
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// The weights of four scores as the two byte planes of 32-bit words: w =
// 256 hi + lo with both bytes signed (w <= 127 * 256).
__device__ inline void pack_weights4(const int32_t* w, int& hi, int& lo)
{
    lo = (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm((uint32_t)w[3], (uint32_t)w[2], 0x0c0c0400u),
                                    __builtin_amdgcn_perm((uint32_t)w[1], (uint32_t)w[0], 0x0c0c0400u),
                                    0x05040100u);
    const uint32_t h0 = (uint32_t)w[0] + 128, h1 = (uint32_t)w[1] + 128, h2 = (uint32_t)w[2] + 128,
                   h3 = (uint32_t)w[3] + 128;
    hi = (int)__builtin_amdgcn_perm(__builtin_amdgcn_perm(h3, h2, 0x0c0c0501u),
                                    __builtin_amdgcn_perm(h1, h0, 0x0c0c0501u), 0x05040100u);
}

// The state of a wave's 16 rows.
template <int KS>
struct Rows {
    double acc[4 * KS][4];  // output channels 16 dt + 4 (lane >> 4) + i of row lane & 15
    double z;
    int32_t m;
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
            if (p.vec) {
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

// One block of 128 positions for the wave's rows.  lo, hi: the row's
// positions (lo, hi] without the sinks; sinks: positions below it are seen too
// (window only).
template <int KS>
__device__ inline void attend_block(const AttnArgs& p, Rows<KS>& st, const v4i (&qh)[KS],
                                    const v4i (&ql)[KS], int32_t cz, int32_t b, int32_t g0,
                                    int64_t blk, int64_t lo, int64_t hi, bool full)
{
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int32_t D = p.kv.D, shift = p.kv.shift;
    const int64_t base = blk * kBlk, psz = (int64_t)1 << shift;
    // pages of the 16-key groups this lane reads keys of (group r >> 2 of each
    // 64) and values of (group g)
    int64_t kp[2], vp[2];
    uint32_t seen = 0xffffffffu;  // keys 64 (i / 16) + 16 g + i % 16 of row r
    bool placed = true;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int64_t ka = base + 64 * h + 16 * (r >> 2), va = base + 64 * h + 16 * g;
        const int64_t kg = kv_page(p.kv, b, ka >> shift), vg = kv_page(p.kv, b, va >> shift);
        if (vg < 0) {
            seen &= ~(0xffffu << (16 * h));
            placed = false;
        }
        kp[h] = ((((kg < 0 ? 0 : kg) * p.kv.G + g0) << shift) + (ka & (psz - 1))) * D;
        vp[h] = ((((vg < 0 ? 0 : vg) * p.kv.G + g0) * D) << shift) + (va & (psz - 1));
    }
    const bool mask = !full || __ballot(!placed) != 0;
    if (mask) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const int64_t j = base + 64 * (i >> 4) + 16 * g + (i & 15);
            if (!(j <= hi && (j > lo || j < p.sinks))) seen &= ~(1u << i);
        }
    }

    // scores
    v4i c[2][4];
    const v4i zero = {0, 0, 0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int8_t* kr = p.kv.k + kp[h] + (4 * j + (r & 3)) * D + 16 * g;
            v4i kf[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s)
                kf[s] = 64 * s + 16 * g < D ? *reinterpret_cast<const v4i*>(kr + 64 * s) : zero;
            v4i a = zero;
#pragma unroll
            for (int s = 0; s < KS; ++s) a = mfma(kf[s], qh[s], a);
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = (int)((uint32_t)a[i] << 8);
            if (cz != 0) {
                const v4i ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};
                v4i k1 = zero;
#pragma unroll
                for (int s = 0; s < KS; ++s) k1 = mfma(kf[s], ones, k1);
#pragma unroll
                for (int i = 0; i < 4; ++i) a[i] += __mul24(k1[i], cz);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) a = mfma(kf[s], ql[s], a);
            c[h][j] = a;
        }
    if (mask) {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (!((seen >> i) & 1)) c[i >> 4][(i >> 2) & 3][i & 3] = kNone;
    }
    int32_t m = kNone;
#pragma unroll
    for (int i = 0; i < 32; ++i) m = max(m, c[i >> 4][(i >> 2) & 3][i & 3]);
    m = max(m, __shfl_xor(m, 16));
    m = max(m, __shfl_xor(m, 32));

    // weights
    v4i wh[2], wl[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            int32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t d = min((uint32_t)m - (uint32_t)c[h][j][i], p.d_cut);
                w[i] = rint_low(exp2_poly(__builtin_fma(-p.tau, (double)d, kLog2One)) + kRintShift);
                if (mask && !((seen >> (16 * h + 4 * j + i)) & 1)) w[i] = 0;
            }
            int hi4, lo4;
            pack_weights4(w, hi4, lo4);
            wh[h][j] = hi4;
            wl[h][j] = lo4;
        }

    // the block joins the rows' state
    const int32_t m_new = max(st.m, m);
    const double f = factor(p, m_new, m);
    if (__ballot(m > st.m) != 0) {
        const double rs = factor(p, m_new, st.m);
        st.z *= rs;
#pragma unroll
        for (int dt = 0; dt < 4 * KS; ++dt)
#pragma unroll
            for (int i = 0; i < 4; ++i) st.acc[dt][i] *= rs;
        st.m = m_new;
    }
    {
        const v4i ones = {0x01010101, 0x01010101, 0x01010101, 0x01010101};
        v4i s = mfma(ones, wh[1], mfma(ones, wh[0], zero));
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = (int)((uint32_t)s[i] << 8);
        s = mfma(ones, wl[1], mfma(ones, wl[0], s));
        st.z = __builtin_fma(f, (double)s[0], st.z);
    }
#pragma unroll
    for (int dt = 0; dt < 4 * KS; ++dt) {
        if (16 * dt >= D) break;
        const int64_t col = (int64_t)(16 * dt + r) << shift;
        const v4i v0 = *reinterpret_cast<const v4i*>(p.kv.v + vp[0] + col);
        const v4i v1 = *reinterpret_cast<const v4i*>(p.kv.v + vp[1] + col);
        v4i s = mfma(v1, wh[1], mfma(v0, wh[0], zero));
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = (int)((uint32_t)s[i] << 8);
        s = mfma(v1, wl[1], mfma(v0, wl[0], s));
#pragma unroll
        for (int i = 0; i < 4; ++i)
            st.acc[dt][i] = __builtin_fma(f, (double)s[i], st.acc[dt][i]);
    }
}

// The code of a row's channel from its sums.
__device__ inline int32_t out_code(const AttnArgs& p, double s, double z)
{
#pragma clang fp contract(off)
    const double v = z > 0.0 ? p.v_scale * (s - (double)p.v_zp * z) / z : 0.0;
    return p.out_bits == 8 ? requant_f64<8>(v, p.out_scale, p.out_zp)
                           : requant_f64<16>(v, p.out_scale, p.out_zp);
}

__device__ inline void store_out(const AttnArgs& p, int64_t t, int32_t head, int32_t d, int32_t q)
{
    const int64_t at = t * p.ldy + (int64_t)head * p.kv.D + d;
    if (p.out_bits == 8) static_cast<int8_t*>(p.y)[at] = (int8_t)q;
    else static_cast<int16_t*>(p.y)[at] = (int16_t)q;
}

// grid (row tiles, G, splits); four waves share a tile's 16 rows and take
// every fourth block of the split.
template <int KS>
__global__ __launch_bounds__(256, 1) void paged_attn_kernel(AttnArgs p)
{
    __shared__ double lds[4][4][64];
    __shared__ double lz[4][kRows];
    __shared__ int32_t lm[4][kRows];
    const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t* starts = p.kv.starts;
    const int32_t grp = p.grp;
    const int64_t tile = blockIdx.x;
    const int32_t b = find_seq(p.kv.B, tile, [=](int32_t i) {
        return (int64_t)starts[i] * grp / kRows + i;
    });
    const int64_t s0 = starts[b], s1 = starts[b + 1], len = p.kv.lens[b];
    if (s0 < 0 || s1 > p.T || s0 >= s1) return;
    const int64_t row0 = (tile - (s0 * grp / kRows + b)) * kRows, rows = (s1 - s0) * grp;
    if (row0 < 0 || row0 >= rows) return;
    const int32_t g0 = blockIdx.y;
    const bool have = row0 + r < rows;
    const int64_t row = have ? row0 + r : rows - 1;
    const int64_t t = s0 + row / grp;
    const int32_t head = g0 * grp + (int32_t)(row % grp);
    // positions seen: (lo, hi], and with a window those below the sinks
    const int64_t hi = len - s1 + t, lo = p.window > 0 ? hi - p.window : -1;

    // blocks that some row of the tile sees: up to the last row's position,
    // with a window from the first row's on, and the sinks'
    const int64_t hi_max = len - s1 + s0 + (min(row0 + kRows, rows) - 1) / grp;
    const int64_t hi_min = len - s1 + s0 + row0 / grp;
    const int64_t list = ((p.kv.ld << p.kv.shift) + kBlk - 1) / kBlk;  // blocks with places
    const int64_t end = hi_max < 0 ? 0 : min(hi_max / kBlk + 1, list);
    int64_t skip0 = 0, skip1 = 0;  // blocks [skip0, skip1) are seen by none
    if (p.window > 0) {
        skip1 = hi_min - p.window + 1 > 0 ? min((hi_min - p.window + 1) / kBlk, end) : 0;
        skip0 = min((p.sinks + kBlk - 1) / kBlk, skip1);
    }
    const int64_t n = end - (skip1 - skip0);
    const int64_t per = (n + p.splits - 1) / p.splits;
    const int64_t i0 = per * blockIdx.z, i1 = min(i0 + per, n);

    Rows<KS> st;
    st.m = kNone;
    st.z = 0.0;
#pragma unroll
    for (int dt = 0; dt < 4 * KS; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) st.acc[dt][i] = 0.0;
    if (i0 < i1) {
        v4i qh[KS], ql[KS];
        int32_t cz;
        load_queries<KS>(p, t, head, have, qh, ql, cz);
        for (int64_t i = i0 + wave; i < i1; i += 4) {
            const int64_t blk = i < skip0 ? i : i + (skip1 - skip0);
            // every row sees all of the block
            const bool full = (blk + 1) * kBlk - 1 <= hi_min &&
                              (p.window == 0 || blk * kBlk > hi_max - p.window);
            attend_block<KS>(p, st, qh, ql, cz, b, g0, blk, lo, hi, full);
        }
    }

    // the four waves' states joined
    if (g == 0) {
        lm[wave][r] = st.m;
        lz[wave][r] = st.z;
    }
    __syncthreads();
    const int32_t m = max(max(lm[0][r], lm[1][r]), max(lm[2][r], lm[3][r]));
    double z = 0.0;
#pragma unroll
    for (int w = 0; w < 4; ++w) z = __builtin_fma(factor(p, m, lm[w][r]), lz[w][r], z);
    const double f = factor(p, m, st.m);
    const int64_t at = (int64_t)blockIdx.z * p.T * p.H + t * p.H + head;
    double* part = p.splits > 1 ? p.part + at * (p.kv.D + 2) : nullptr;
    if (part && have && wave == 0 && g == 0) {
        part[p.kv.D] = z;
        part[p.kv.D + 1] = (double)m;
    }
#pragma unroll
    for (int dt = 0; dt < 4 * KS; ++dt) {
        if (16 * dt >= p.kv.D) break;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) lds[wave][i][lane] = f * st.acc[dt][i];
        __syncthreads();
        const double s = (lds[0][wave][lane] + lds[1][wave][lane]) +
                         (lds[2][wave][lane] + lds[3][wave][lane]);
        if (!have) continue;
        const int32_t d = 16 * dt + 4 * g + wave;
        if (part) part[d] = s;
        else store_out(p, t, head, d, out_code(p, s, z));
    }
}

// One wave per row joins the splits.
__global__ __launch_bounds__(256) void paged_attn_join_kernel(AttnArgs p)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= p.T * p.H) return;
    const int64_t t = row / p.H;
    const int32_t b = find_seq(p.kv.B, t, [=](int32_t i) { return (int64_t)p.kv.starts[i]; });
    if (t < p.kv.starts[b] || t >= p.kv.starts[b + 1]) return;
    const int32_t D = p.kv.D;
    const int64_t step = p.T * p.H * (D + 2);
    const double* part = p.part + row * (D + 2);
    double m = (double)kNone;
    for (int s = 0; s < p.splits; ++s) m = fmax(m, part[s * step + D + 1]);
    double z = 0.0, acc[4] = {0.0, 0.0, 0.0, 0.0};
    for (int s = 0; s < p.splits; ++s) {
        const double* x = part + s * step;
        const double f = exp2_poly(fmax(-p.tau * (m - x[D + 1]), -1100.0));
        z = __builtin_fma(f, x[D], z);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (lane + 64 * i < D) acc[i] = __builtin_fma(f, x[lane + 64 * i], acc[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < D)
            store_out(p, t, (int32_t)(row % p.H), lane + 64 * i, out_code(p, acc[i], z));
}

// Row tiles of all sequences, at most.
int64_t row_tiles(int64_t T, int64_t B, int32_t grp) { return T * grp / kRows + B; }

// Parts the keys of every tile are split into: enough work-groups for the
// chip, at least four blocks each.
int64_t split_count(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D, int64_t max_len)
{
    const int64_t groups = row_tiles(T, B, H / G) * G;
    int64_t s = 1024 / (groups > 0 ? groups : 1);
    const int64_t blocks = (max_len + kBlk - 1) / kBlk;
    s = std::min(s, (blocks + 3) / 4);
    s = std::min<int64_t>(s, MQ_ATTN_MAX_WORKSPACE / (T * H * (D + 2) * 8));
    return s < 1 ? 1 : s;
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
    p.tau = sigma * 1.4426950408889634;  // log2(e)
    p.v_scale = v_scale;
    p.out_scale = out_scale;
    // a weight is 0 below 2^-1: from 2^-40 of the largest on, whatever the
    // distance
    const double cut = 40.0 / p.tau;
    p.d_cut = cut < 4294967295.0 ? (uint32_t)std::ceil(cut) : 0xFFFFFFFFu;
    p.window = window;
    p.sinks = window > 0 ? sinks : 0;
    p.vec = ((uintptr_t)q % 16) == 0 && ldq % 8 == 0;
    int64_t splits = split_count(T, kv.B, H, kv.G, kv.D, max_len);
    const int64_t one = T * H * (kv.D + 2) * 8;
    if (!ws) splits = 1;
    splits = std::min(splits, std::max<int64_t>(ws_bytes / one, 1));
    p.splits = (int32_t)splits;
    p.part = static_cast<double*>(ws);
    const dim3 grid((unsigned)row_tiles(T, kv.B, p.grp), (unsigned)kv.G, (unsigned)splits);
    switch ((kv.D + 63) / 64) {
    case 1: paged_attn_kernel<1><<<grid, 256, 0, s>>>(p); break;
    case 2: paged_attn_kernel<2><<<grid, 256, 0, s>>>(p); break;
    case 3: paged_attn_kernel<3><<<grid, 256, 0, s>>>(p); break;
    default: paged_attn_kernel<4><<<grid, 256, 0, s>>>(p); break;
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || splits == 1) return e;
    paged_attn_join_kernel<<<(unsigned)((T * H + 3) / 4), 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mq
