// Appending a batch's new tokens to the paged key/value cache: rotation and
// requantization of queries and keys by each token's own position, the
// values transposed into their pages.
#include "codes.h"
#include "kvcache.h"
#include "mq_internal.h"

namespace mq {
namespace {

struct AppendArgs {
    KvArgs kv;
    const int16_t* q;
    const int16_t* k;
    const int8_t* v;
    int16_t* q_out;
    const double* angles;  // or nullptr
    int64_t ldq, ldk, ldv, ldo, positions, T;
    float aq, aqo, ak, ako;
    int32_t zq, zqo, zk, zko;
    int32_t H;
    int32_t chunks;    // blocks per token of the rotation
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

// NP neighbouring pairs (i, i + D/2) of one head of the row x -> codes r.
template <int BITS, int NP>
__device__ inline void rotate(const int16_t* x, int32_t half, int32_t i, float ax, int32_t zx,
                              const double* cs, float ay, int32_t zy, int32_t* r)
{
#pragma clang fp contract(off)
    int32_t c0[NP], c1[NP];
    if constexpr (NP == 8) {
        unpack8(*reinterpret_cast<const v4i*>(x + i), c0);
        unpack8(*reinterpret_cast<const v4i*>(x + i + half), c1);
    } else {
        c0[0] = x[i];
        c1[0] = x[i + half];
    }
    const double ri = 1.0 / (double)ay;
    double w[2 * NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) {
        const double f0 = (double)ax * (double)(c0[k] - zx);
        const double f1 = (double)ax * (double)(c1[k] - zx);
        if (cs) {
            const double c = cs[2 * (i + k)], sn = cs[2 * (i + k) + 1];
            w[k] = f0 * c - f1 * sn;
            w[NP + k] = f1 * c + f0 * sn;
        } else {
            w[k] = f0;
            w[NP + k] = f1;
        }
    }
    requant_codes<BITS, 2 * NP>(r, zy, [&](int k) { return w[k] / (double)ay; },
                                [&](int k) { return w[k] * ri; });
}

template <int NP>
__device__ inline void rotation_block(const AppendArgs& p, int64_t blk)
{
    const int64_t t = blk / p.chunks;
    int32_t b;
    int64_t pos;
    if (!token_place(p, t, b, pos)) return;
    const int32_t half = p.kv.D / 2, per = half / NP;
    int32_t u = (int32_t)(blk - t * p.chunks) * 256 + (int32_t)threadIdx.x;
    const double* cs = p.angles ? p.angles + pos * p.kv.D : nullptr;
    int32_t r[2 * NP];
    if (u < p.H * per) {
        const int32_t h = u / per, i = (u - h * per) * NP;
        rotate<16, NP>(p.q + t * p.ldq + (int64_t)h * p.kv.D, half, i, p.aq, p.zq, cs, p.aqo,
                       p.zqo, r);
        int16_t* y = p.q_out + t * p.ldo + (int64_t)h * p.kv.D;
        if constexpr (NP == 8) {
            store8<16>(y, i, r);
            store8<16>(y, i + half, r + NP);
        } else {
            y[i] = (int16_t)r[0];
            y[i + half] = (int16_t)r[1];
        }
        return;
    }
    u -= p.H * per;
    if (u >= p.kv.G * per) return;
    const int64_t pg = kv_page(p.kv, b, pos >> p.kv.shift);
    if (pg < 0) return;
    const int32_t g = u / per, i = (u - g * per) * NP;
    rotate<8, NP>(p.k + t * p.ldk + (int64_t)g * p.kv.D, half, i, p.ak, p.zk, cs, p.ako, p.zko,
                  r);
    const int64_t slot = pos & (((int64_t)1 << p.kv.shift) - 1);
    int8_t* y = p.kv.k + ((((pg * p.kv.G + g) << p.kv.shift) + slot) * p.kv.D);
    if constexpr (NP == 8) {
        store8<8>(y, i, r);
        store8<8>(y, i + half, r + NP);
    } else {
        y[i] = (int8_t)r[0];
        y[i + half] = (int8_t)r[1];
    }
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

template <int NP>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs p)
{
    const int64_t blk = blockIdx.x;
    if (blk < p.rot) rotation_block<NP>(p, blk);
    else value_block(p, blk - p.rot);
}

}  // namespace

hipError_t launch_rope_append(const KvArgs& kv, const int16_t* q, int64_t ldq, const int16_t* k,
                              int64_t ldk, const int8_t* v, int64_t ldv, int64_t T, int32_t H,
                              float aq, int32_t zq, float aqo, int32_t zqo, float ak, int32_t zk,
                              float ako, int32_t zko, const double* angles, int64_t positions,
                              int16_t* q_out, int64_t ldo, hipStream_t s)
{
    AppendArgs p{kv, q, k, v, q_out, angles, ldq, ldk, ldv, ldo, positions, T, aq, aqo, ak, ako,
                 zq, zqo, zk, zko, H, 0, 0, 0};
    const bool vec = ((uintptr_t)q % 16) == 0 && ((uintptr_t)k % 16) == 0 &&
                     ((uintptr_t)q_out % 16) == 0 && ldq % 8 == 0 && ldk % 8 == 0 && ldo % 8 == 0;
    const int64_t pairs = (int64_t)(H + kv.G) * (kv.D / 2) / (vec ? 8 : 1);
    p.chunks = (int32_t)((pairs + 255) / 256);
    p.rot = T * p.chunks;
    p.v_chunks = (kv.G * kv.D + 255) / 256;
    const int64_t tiles = T / 16 + 2 * (int64_t)kv.B;
    const int64_t blocks = p.rot + tiles * p.v_chunks;
    if (blocks > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (vec) rope_append_kernel<8><<<(unsigned)blocks, 256, 0, s>>>(p);
    else rope_append_kernel<1><<<(unsigned)blocks, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace mq
