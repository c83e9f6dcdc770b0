// Appending a batch's new tokens to the paged key/value cache: rotation and
// requantization of queries and keys by each token's own position, the
// values transposed into their pages.
//
// Memory bounds it at many tokens, the way to a token's place (its sequence,
// then the length, then angles and page: each waits for the one before) at
// few.  A wave rotates all heads of a token, so that the angles are read and
// scaled once and each lane keeps its pairs' in registers; of few tokens
// several waves share the heads, up to 4096 waves in all.  32 heads of 64, 4 of
// the cache, us: 1 token 3.3 (one wave per token: 5.1), 250 sequences' one token
// each 5.8 (7.5), 4740 tokens 15.9 for 45 MB (five waves per token 27, a
// block per token 22).
#include <algorithm>

#include "codes.h"
#include "kvcache.h"
#include "mq_internal.h"

namespace mq {
namespace {

constexpr int kPairs = 4;  // pairs of a lane

// Codes of scale ax and zero-point zx to codes of scale ay and zero-point zy.
struct Format {
    float ax, ay;
    int32_t zx, zy;
    double ratio;  // ax / ay, to three roundings
};

struct AppendArgs {
    KvArgs kv;
    const int16_t* q;
    const int16_t* k;
    const int8_t* v;
    int16_t* q_out;
    const double* angles;  // or nullptr
    int64_t ldq, ldk, ldv, ldo, positions, T;
    Format fq, fk;
    int32_t H;
    int32_t waves;     // per token of the rotation
    int32_t per_turn;  // heads that a wave rotates at once
    int32_t inv_per;   // 2^16 / lanes per head, rounded up
    int32_t k_first;   // the wave with the first of the keys' turns
    int64_t rot;       // blocks of the rotation; the values' follow
    int32_t v_chunks;  // blocks per 16 positions of the values
};

// The place of token row t: its sequence and position; false if it belongs to
// no sequence or has no angle.
__device__ inline bool token_place(const AppendArgs& p, int64_t t, int32_t& b, int64_t& pos)
{
    const int32_t* st = p.kv.starts;
    b = find_seq(p.kv.B, t, [=](int32_t i) { return (int64_t)st[i]; });
    const int64_t s0 = st[b], s1 = st[b + 1];
    if (t < s0 || t >= s1) return false;
    pos = (int64_t)p.kv.lens[b] - s1 + t;
    return pos >= 0 && (!p.angles || pos < p.positions);
}

// Neighbouring pairs (i, i + D/2) of a head, c0 and c1 its codes there, ->
// codes r.  c and sn: cos and sin of the pairs times f.ratio; cs: cos and sin
// (nullptr: no rotation); large: one of c or sn is over 4 or NaN.
//
// A pair takes two products and two fused ones.  |n| < 2^16, so for |c|, |sn|
// <= 4 the terms are below 2^18 and their eight roundings (three of c's or
// sn's, a product's and a sum's here, a product's, a sum's and a quotient's in
// the definition) move the result by less than 2^-31: where it is further than
// 2^-30 from every half-integer, both round to the same integer.  A wave with a
// result nearer than that, or with larger c or sn, evaluates the definition.
template <int BITS>
__device__ __forceinline__ void rotate(const int32_t (&c0)[kPairs], const int32_t (&c1)[kPairs],
                                       const double (&c)[kPairs], const double (&sn)[kPairs],
                                       const double* cs, bool large, const Format& f,
                                       int32_t (&r)[2 * kPairs])
{
#pragma clang fp contract(off)
    double far = 0.0;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        const double n0 = (double)(c0[k] - f.zx), n1 = (double)(c1[k] - f.zx);
        const double t0 = __builtin_fma(n0, c[k], -(n1 * sn[k]));
        const double t1 = __builtin_fma(n1, c[k], n0 * sn[k]);
        const double r0 = t0 + kRintShift, r1 = t1 + kRintShift;
        r[k] = rint_low(r0);
        r[kPairs + k] = rint_low(r1);
        far = fmax(far, fabs(t0 - (r0 - kRintShift)));
        far = fmax(far, fabs(t1 - (r1 - kRintShift)));
    }
    if (__builtin_expect(__ballot(large || far > 0.5 - 0x1p-30) != 0, 0)) {
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const double ck = cs ? cs[2 * k] : 1.0, sk = cs ? cs[2 * k + 1] : 0.0;
            const double f0 = (double)f.ax * (double)(c0[k] - f.zx);
            const double f1 = (double)f.ax * (double)(c1[k] - f.zx);
            const double w0 = f0 * ck - f1 * sk, w1 = f1 * ck + f0 * sk;
            r[k] = rint_low(limit_quotient(w0 / (double)f.ay) + kRintShift);
            r[kPairs + k] = rint_low(limit_quotient(w1 / (double)f.ay) + kRintShift);
            __builtin_amdgcn_sched_barrier(0);  // one pair's registers at a time
        }
    }
#pragma unroll
    for (int k = 0; k < 2 * kPairs; ++k) r[k] = clamp_code<BITS>(r[k] + f.zy);
}

// Four codes of a row: one access of 8 or 4 bytes where rows are aligned.
template <bool VEC>
__device__ __forceinline__ int2 load4(const int16_t* x)
{
    if constexpr (VEC) return *reinterpret_cast<const int2*>(x);
    return make_int2((uint16_t)x[0] | (int)((uint32_t)(uint16_t)x[1] << 16),
                     (uint16_t)x[2] | (int)((uint32_t)(uint16_t)x[3] << 16));
}
template <bool VEC>
__device__ __forceinline__ void store4(int16_t* y, const int32_t* r)
{
    if constexpr (VEC) {
        *reinterpret_cast<int2*>(y) =
            make_int2((r[0] & 0xffff) | (int)((uint32_t)r[1] << 16),
                      (r[2] & 0xffff) | (int)((uint32_t)r[3] << 16));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) y[k] = (int16_t)r[k];
    }
}
template <bool VEC>
__device__ __forceinline__ void store4(int8_t* y, const int32_t* r)  // cache rows are aligned
{
    *reinterpret_cast<uint32_t*>(y) = ((uint32_t)r[0] & 255) | ((uint32_t)r[1] & 255) << 8 |
                                      ((uint32_t)r[2] & 255) << 16 | (uint32_t)r[3] << 24;
}

// The heads of one token that a wave rotates: D / 8 lanes per head, so many
// heads at once, in turns first, first + step, ... of `turns`.
struct Turns {
    int32_t head, i, per;  // this lane's head of a turn (64: none) and first pair
    int32_t first, step;
};
constexpr int kAhead = 2;  // turns whose codes are under way
template <bool VEC>
__device__ __forceinline__ void load_turn(const int16_t* x, int32_t heads, int32_t D, const Turns& w,
                                          int32_t turn, int2 (&v)[2])
{
    // (heads past the last: the last one's)
    const int16_t* at = x + (int64_t)min(turn * w.per + w.head, heads - 1) * D + w.i;
    v[0] = load4<VEC>(at);
    v[1] = load4<VEC>(at + D / 2);
}
template <int BITS, bool VEC, class Out>
__device__ __forceinline__ void rotate_heads(const int16_t* x, int32_t heads, int32_t D,
                                             const Turns& w, int2 (&next)[kAhead][2],
                                             const double* cs, const Format& f, Out out)
{
    double c[kPairs], sn[kPairs];
    bool large = false;
#pragma unroll
    for (int k = 0; k < kPairs; ++k) {
        c[k] = cs ? cs[2 * k] * f.ratio : f.ratio;
        sn[k] = cs ? cs[2 * k + 1] * f.ratio : 0.0;
        large |= !(fabs(c[k]) <= 4.0 && fabs(sn[k]) <= 4.0);
    }
#pragma unroll 1
    for (int32_t turn = w.first; turn * w.per < heads; turn += kAhead * w.step)
#pragma unroll
        for (int n = 0; n < kAhead; ++n) {
            const int32_t now = turn + n * w.step, h = now * w.per + w.head;
            if (now * w.per >= heads) break;
            int32_t c0[kPairs], c1[kPairs], r[2 * kPairs];
            c0[0] = (int16_t)next[n][0].x;
            c0[1] = next[n][0].x >> 16;
            c0[2] = (int16_t)next[n][0].y;
            c0[3] = next[n][0].y >> 16;
            c1[0] = (int16_t)next[n][1].x;
            c1[1] = next[n][1].x >> 16;
            c1[2] = (int16_t)next[n][1].y;
            c1[3] = next[n][1].y >> 16;
            if ((now + kAhead * w.step) * w.per < heads)
                load_turn<VEC>(x, heads, D, w, now + kAhead * w.step, next[n]);
            rotate<BITS>(c0, c1, c, sn, cs, large, f, r);
            if (w.head < w.per && h < heads) {
                auto y = out(h) + w.i;
                store4<VEC>(y, r);
                store4<VEC>(y + D / 2, r + kPairs);
            }
        }
}

// A token's heads in one wave or, of few tokens, in several.
template <bool VEC>
__device__ inline void rotation_wave(const AppendArgs& p, int64_t id)
{
    // (one wave per token, or a few thousand waves in all)
    const int64_t t = p.waves == 1 ? id : (uint32_t)id / (uint32_t)p.waves;
    if (t >= p.T) return;
    const int lane = threadIdx.x & 63;
    const int32_t D = p.kv.D, per = D / 2 / kPairs;
    Turns w;
    w.per = p.per_turn;
    w.head = (lane * p.inv_per) >> 16;  // lane / per
    w.i = (lane - w.head * per) * kPairs;
    w.step = p.waves;
    w.first = (int32_t)(id - t * p.waves);
    Turns wk = w;  // the keys' turns follow the queries'
    wk.first = w.first - p.k_first + (w.first < p.k_first ? p.waves : 0);
    int32_t b;
    int64_t pos;
    if (!token_place(p, t, b, pos)) return;
    const int16_t* q = p.q + t * p.ldq;
    const int16_t* k = p.k + t * p.ldk;
    int2 qn[kAhead][2], kn[kAhead][2];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) {
        if ((w.first + n * w.step) * w.per < p.H)
            load_turn<VEC>(q, p.H, D, w, w.first + n * w.step, qn[n]);
        if ((wk.first + n * w.step) * w.per < p.kv.G)
            load_turn<VEC>(k, p.kv.G, D, wk, wk.first + n * w.step, kn[n]);
    }
    const double* cs = p.angles ? p.angles + pos * D + 2 * w.i : nullptr;
    int16_t* y = p.q_out + t * p.ldo;
    if (w.first * w.per < p.H)
        rotate_heads<16, VEC>(q, p.H, D, w, qn, cs, p.fq, [=](int32_t h) { return y + (int64_t)h * D; });
    if (wk.first * w.per >= p.kv.G) return;
    const int64_t pg = kv_page(p.kv, b, pos >> p.kv.shift);
    if (pg < 0) return;
    const int64_t slot = pos & (((int64_t)1 << p.kv.shift) - 1);
    int8_t* kc = p.kv.k + (((pg * p.kv.G) << p.kv.shift) + slot) * D;
    const int64_t head = (int64_t)D << p.kv.shift;
    rotate_heads<8, VEC>(k, p.kv.G, D, wk, kn, cs, p.fk, [=](int32_t h) { return kc + h * head; });
}

// Tiles of 16 aligned positions of one sequence, a thread per channel: 16
// neighbouring slots of a channel are 16 contiguous bytes of the cache.
__device__ inline void value_block(const AppendArgs& p, int64_t blk)
{
    const int64_t tile = blk / p.v_chunks;
    const int32_t* st = p.kv.starts;
    const int32_t b =
        find_seq(p.kv.B, tile, [=](int32_t i) { return (int64_t)(st[i] >> 4) + 2 * (int64_t)i; });
    const int64_t s0 = st[b], s1 = st[b + 1], len = p.kv.lens[b];
    if (s0 < 0 || s1 > p.T || s0 >= s1) return;
    const int64_t local = tile - ((s0 >> 4) + 2 * (int64_t)b);
    if (local < 0) return;
    // positions [lo, hi) have rows; row of position x: s1 - len + x
    int64_t lo = len - (s1 - s0), hi = len;
    if (lo < 0) lo = 0;
    if (p.angles && hi > p.positions) hi = p.positions;
    const int64_t x0 = ((lo >> 4) + local) << 4;
    if (x0 >= hi) return;
    const int64_t pg = kv_page(p.kv, b, x0 >> p.kv.shift);
    if (pg < 0) return;
    const int32_t c = (int32_t)(blk - tile * p.v_chunks) * 256 + (int32_t)threadIdx.x;
    if (c >= p.kv.G * p.kv.D) return;
    const int64_t slot = x0 & (((int64_t)1 << p.kv.shift) - 1);
    int8_t* y = p.kv.v + (((pg * p.kv.G * p.kv.D + c) << p.kv.shift) + slot);
    const int8_t* x = p.v + (s1 - len + x0) * p.ldv + c;
    if (x0 >= lo && x0 + 16 <= hi) {
        v4i w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t d = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                d |= (uint32_t)(uint8_t)x[(int64_t)(4 * i + j) * p.ldv] << (8 * j);
            w[i] = (int)d;
        }
        *reinterpret_cast<v4i*>(y) = w;
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (x0 + j >= lo && x0 + j < hi) y[j] = x[(int64_t)j * p.ldv];
    }
}

template <bool VEC>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs p)
{
    const int64_t blk = blockIdx.x;
    if (blk < p.rot)
        rotation_wave<VEC>(
            p, 4 * blk + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6));
    else
        value_block(p, blk - p.rot);
}

}  // namespace

hipError_t launch_rope_append(const KvArgs& kv, const int16_t* q, int64_t ldq, const int16_t* k,
                              int64_t ldk, const int8_t* v, int64_t ldv, int64_t T, int32_t H,
                              float aq, int32_t zq, float aqo, int32_t zqo, float ak, int32_t zk,
                              float ako, int32_t zko, const double* angles, int64_t positions,
                              int16_t* q_out, int64_t ldo, hipStream_t s)
{
    AppendArgs p;
    p.kv = kv;
    p.q = q;
    p.k = k;
    p.v = v;
    p.q_out = q_out;
    p.angles = angles;
    p.ldq = ldq;
    p.ldk = ldk;
    p.ldv = ldv;
    p.ldo = ldo;
    p.positions = positions;
    p.T = T;
    p.H = H;
    p.fq = Format{aq, aqo, zq, zqo,
                  (double)aq * (1.0 / (double)aqo)};
    p.fk = Format{ak, ako, zk, zko,
                  (double)ak * (1.0 / (double)ako)};
    const bool vec = ((uintptr_t)q % 8) == 0 && ((uintptr_t)k % 8) == 0 &&
                     ((uintptr_t)q_out % 8) == 0 && ldq % 4 == 0 && ldk % 4 == 0 && ldo % 4 == 0;
    const int32_t per = kv.D / 2 / kPairs;
    p.per_turn = 64 / per;
    p.inv_per = (65536 + per - 1) / per;
    const int32_t q_turns = (H + p.per_turn - 1) / p.per_turn;
    const int32_t turns = q_turns + (kv.G + p.per_turn - 1) / p.per_turn;
    p.waves = (int32_t)std::max<int64_t>(1, std::min<int64_t>(turns, 4096 / T));
    p.k_first = q_turns % p.waves;
    p.rot = (T * p.waves + 3) / 4;
    p.v_chunks = (kv.G * kv.D + 255) / 256;
    const int64_t tiles = T / 16 + 2 * (int64_t)kv.B;
    const int64_t blocks = p.rot + tiles * p.v_chunks;
    if (blocks >= kMaxBlocks) return hipErrorInvalidConfiguration;
    if (vec) rope_append_kernel<true><<<(unsigned)blocks, 256, 0, s>>>(p);
    else rope_append_kernel<false><<<(unsigned)blocks, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mq
