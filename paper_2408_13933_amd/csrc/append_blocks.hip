// Appending a batch's new tokens to the cache with block scales: queries and
// keys rotated by their positions' angles (fp64, then rounded once to fp32),
// keys and values quantized by the largest magnitude of their block and head.
//
// A work item is one aligned block of one sequence and head, of the keys or of
// the values: its new elements' maximum, the scale, the codes, and the codes it
// held before by the new scale where that is larger.  Nobody else writes the
// block, so nothing waits for anything.  Memory bounds it at many tokens, the
// way to a token's place (sequence, length, page list, old scale) at few: five prompts of
// 450 to 900 tokens (32 and 4 heads of 64, fp16) 12.2 us, one token of each of 250
// sequences (8 heads and one of 256, bf16) 8.0.
#include <algorithm>

#include "kvblocks.h"
#include "mq_internal.h"
#include "tokens.h"
#include "wave.h"

namespace mq {
namespace {

constexpr int kPairs = 4;  // pairs of a lane's chunk
constexpr int kHold = 4;   // key chunks that a lane holds between maximum and codes

struct AppendArgs {
    BlockCache c;
    const void* q;
    const void* k;
    const void* v;
    void* q_out;
    const double* angles;  // or nullptr
    int64_t ldq, ldk, ldv, ldo, positions, T;
    int32_t H;
    int32_t waves;     // per token of the queries' rotation
    int32_t per_turn;  // heads that a wave rotates at once
    uint32_t inv_per;  // 2^32 / (D / 8), rounded up
    uint32_t inv_half; // 2^32 / (D / 2), rounded up
    int64_t rot;       // blocks of the queries' rotation; the items' follow
    int64_t items;
};

// x / d by inv = 2^32 / d rounded up (x d < 2^32)
__device__ inline int32_t div_by(int32_t x, uint32_t inv) { return (int32_t)__umulhi((uint32_t)x, inv); }

// Four consecutive elements as fp32.
template <int TYPE, bool VEC>
struct Four {
    uint32_t d[TYPE == MQ_F32 ? 4 : 2];
    __device__ void load(const void* x, int64_t i)
    {
        if constexpr (TYPE == MQ_F32) {
            const uint32_t* p = static_cast<const uint32_t*>(x) + i;
            if constexpr (VEC) {
                const uint4 v = *reinterpret_cast<const uint4*>(p);
                d[0] = v.x, d[1] = v.y, d[2] = v.z, d[3] = v.w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) d[j] = p[j];
            }
        } else {
            const uint16_t* p = static_cast<const uint16_t*>(x) + i;
            if constexpr (VEC) {
                const uint2 v = *reinterpret_cast<const uint2*>(p);
                d[0] = v.x, d[1] = v.y;
            } else {
                d[0] = p[0] | (uint32_t)p[1] << 16;
                d[1] = p[2] | (uint32_t)p[3] << 16;
            }
        }
    }
    __device__ float operator[](int i) const
    {
        if constexpr (TYPE == MQ_F32) return __builtin_bit_cast(float, d[i]);
        else return half_of<TYPE>(d[i >> 1], i & 1);
    }
};
template <int TYPE, bool VEC>
__device__ inline void store_four(void* y, int64_t i, const float* r)
{
    if constexpr (TYPE == MQ_F32) {
        float* p = static_cast<float*>(y) + i;
        if constexpr (VEC) {
            *reinterpret_cast<float4*>(p) = make_float4(r[0], r[1], r[2], r[3]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j] = r[j];
        }
    } else {
        const uint32_t a = pack2<TYPE>(r[0], r[1]), b = pack2<TYPE>(r[2], r[3]);
        uint16_t* p = static_cast<uint16_t*>(y) + i;
        if constexpr (VEC) {
            *reinterpret_cast<uint2*>(p) = make_uint2(a, b);
        } else {
            p[0] = (uint16_t)a, p[1] = (uint16_t)(a >> 16);
            p[2] = (uint16_t)b, p[3] = (uint16_t)(b >> 16);
        }
    }
}

// cos and sin of a chunk's pairs.
struct Angles {
    double c[kPairs], s[kPairs];
    __device__ void load(const double* a)
    {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            const double2 v = reinterpret_cast<const double2*>(a)[i];
            c[i] = v.x;
            s[i] = v.y;
        }
    }
};

// The chunk's pairs (u, w) turned: u cos - w sin, w cos + u sin, in fp64 without
// fused steps, so that fp32 values and codes do not depend on how they are made.
template <class F>
__device__ inline void turn(const F& u, const F& w, const Angles& a, bool have, float (&r)[8])
{
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < kPairs; ++i) {
        const double x = (double)u[i], y = (double)w[i];
        r[i] = have ? (float)(x * a.c[i] - y * a.s[i]) : u[i];
        r[4 + i] = have ? (float)(y * a.c[i] + x * a.s[i]) : w[i];
    }
}

// The largest finite magnitude.
__device__ inline uint32_t finite_bits(float x)
{
    const uint32_t b = abs_bits(x);
    return b < kInfBits ? b : 0;
}

// rint(x inv) limited to +-127 (infinities), NaN to 0; low byte.
__device__ inline uint32_t block_code(float x, float inv)
{
    const float v = fminf(fmaxf(x * inv, -127.0f), 127.0f);
    return x == x ? __builtin_bit_cast(uint32_t, v + 12582912.0f) : 0u;
}
// A code by a larger scale.
__device__ inline uint32_t code_again(int32_t c, float ratio)
{
    return __builtin_bit_cast(uint32_t, (float)c * ratio + 12582912.0f);
}
__device__ inline uint32_t codes_again(uint32_t d, float ratio)
{
    return pack_codes(code_again((int8_t)d, ratio), code_again((int8_t)(d >> 8), ratio),
                      code_again((int8_t)(d >> 16), ratio), code_again((int8_t)(d >> 24), ratio));
}

// The queries of one token in one wave or, of few tokens, in several.
template <int TYPE, bool VEC>
__device__ inline void rotate_queries(const AppendArgs& p, int64_t id)
{
    const KvArgs& kv = p.c.kv;
    const int64_t t = p.waves == 1 ? id : (uint32_t)id / (uint32_t)p.waves;
    if (t >= p.T) return;
    const int32_t* st = kv.starts;
    const int32_t b = find_seq(kv.B, t, [=](int32_t i) { return (int64_t)st[i]; });
    const int64_t s0 = st[b], s1 = st[b + 1];
    if (t < s0 || t >= s1) return;
    const int64_t pos = (int64_t)kv.lens[b] - s1 + t;
    if (pos < 0 || (p.angles && pos >= p.positions)) return;
    const int lane = threadIdx.x & 63;
    const int32_t D = kv.D, per = D / 8;
    const int32_t head = div_by(lane, p.inv_per), i = (lane - head * per) * kPairs;
    if (head >= p.per_turn) return;
    Angles a;
    if (p.angles) a.load(p.angles + pos * D + 2 * i);
    constexpr int U = 4;  // turns whose reads are under way together
    const int32_t step = p.waves * p.per_turn;
    for (int32_t h0 = (int32_t)(id - t * p.waves) * p.per_turn + head; h0 < p.H; h0 += U * step) {
        Four<TYPE, VEC> u[U], w[U];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int64_t at = t * p.ldq + (int64_t)min(h0 + j * step, p.H - 1) * D + i;
            u[j].load(p.q, at);
            w[j].load(p.q, at + D / 2);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int32_t h = h0 + j * step;
            if (h >= p.H) break;
            float r[8];
            turn(u[j], w[j], a, p.angles != nullptr, r);
            const int64_t to = t * p.ldo + (int64_t)h * D + i;
            store_four<TYPE, VEC>(p.q_out, to, r);
            store_four<TYPE, VEC>(p.q_out, to + D / 2, r + 4);
        }
    }
}

// One block of one sequence and head.
struct Item {
    int64_t pg;       // its page
    int32_t g, slot;  // head, first slot in the page
    int64_t x0;       // its first position
    int32_t lo, hi;   // positions that the call writes, from x0 on
    int64_t row;      // token row of position x0
    bool values;
};

// The index counts, per sequence, from floor(starts[b] / block) + 2 b: an upper
// bound of the blocks before it that needs no scan.  Uniform.
__device__ inline bool find_item(const AppendArgs& p, int64_t id, Item& it)
{
    const KvArgs& kv = p.c.kv;
    const int32_t G2 = 2 * kv.G;
    const int64_t tile = id / G2;
    const int32_t part = (int32_t)(id - tile * G2);
    it.values = part >= kv.G;
    it.g = it.values ? part - kv.G : part;
    const int32_t* st = kv.starts;
    const int sh = p.c.bshift;
    const int32_t b =
        find_seq(kv.B, tile, [=](int32_t i) { return (int64_t)(st[i] >> sh) + 2 * (int64_t)i; });
    const int64_t s0 = st[b], s1 = st[b + 1], len = kv.lens[b];
    if (s0 < 0 || s1 > p.T || s0 >= s1) return false;
    const int64_t local = tile - ((s0 >> sh) + 2 * (int64_t)b);
    if (local < 0) return false;
    int64_t lo = len - (s1 - s0), hi = len;
    if (lo < 0) lo = 0;
    if (p.angles && hi > p.positions) hi = p.positions;
    const int64_t x0 = ((lo >> sh) + local) << sh;
    if (x0 >= hi) return false;
    it.pg = kv_page(kv, b, x0 >> kv.shift);
    if (it.pg < 0) return false;
    it.slot = (int32_t)(x0 & (((int64_t)1 << kv.shift) - 1));
    it.x0 = x0;
    it.lo = (int32_t)(lo > x0 ? lo - x0 : 0);
    it.hi = (int32_t)(hi - x0 < (1 << sh) ? hi - x0 : 1 << sh);
    it.row = s1 - len + x0;
    return true;
}

// The scale of a block from its new elements' largest magnitude and, where it
// holds tokens before them, its old scale; ratio: by what those codes change.
struct Scale {
    float s, inv, ratio;
    bool again;
    __device__ Scale(uint32_t most, bool held, float before)
    {
        const float old = held && before > 0.0f && abs_bits(before) < kInfBits ? before : 0.0f;
        s = fmaxf(old, scale_of(most));
        inv = 1.0f / s;
        ratio = old / s;
        again = held && !(before == s);
    }
};

template <int WAVES>
__device__ inline uint32_t item_max(uint32_t v, uint32_t* lds)
{
    v = wave_max(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
    }
    return v;
}

template <int TYPE, bool VEC, int WAVES>
__device__ inline void key_item(const AppendArgs& p, const Item& it, uint32_t* lds)
{
    constexpr int T = 64 * WAVES;
    const int t = WAVES == 1 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
    const int32_t D = p.c.kv.D, per = D / 8, n = (it.hi - it.lo) * per;
    float* scale = p.c.k_scale + scale_at(p.c, it.pg, it.g, it.slot);
    const float before = it.lo > 0 ? *scale : 0.0f;
    int8_t* y = p.c.kv.k + (((it.pg * p.c.kv.G + it.g) << p.c.kv.shift) + it.slot) * D;
    struct Chunk {
        Four<TYPE, VEC> u, w;
        Angles a;
    };
    auto load = [&](int32_t i, Chunk& c) {
        const int32_t tok = div_by(i, p.inv_per), e = (i - tok * per) * kPairs;
        const int32_t x = it.lo + tok;
        const int64_t at = (it.row + x) * p.ldk + (int64_t)it.g * D + e;
        c.u.load(p.k, at);
        c.w.load(p.k, at + D / 2);
        if (p.angles) c.a.load(p.angles + (it.x0 + x) * D + 2 * e);
    };
    auto most_of = [](const float (&r)[8], uint32_t m) {
#pragma unroll
        for (int j = 0; j < 8; ++j) m = max(m, finite_bits(r[j]));
        return m;
    };
    auto store = [&](int32_t i, const float (&r)[8], float inv) {
        const int32_t tok = div_by(i, p.inv_per), e = (i - tok * per) * kPairs;
        uint32_t* to = reinterpret_cast<uint32_t*>(y + (it.lo + tok) * D + e);
        to[0] = pack_codes(block_code(r[0], inv), block_code(r[1], inv), block_code(r[2], inv),
                           block_code(r[3], inv));
        to[D / 8] = pack_codes(block_code(r[4], inv), block_code(r[5], inv),
                               block_code(r[6], inv), block_code(r[7], inv));
    };
    float r[kHold][8];
    uint32_t most = 0;
    const bool turned = p.angles != nullptr;
    {
        Chunk c[kHold];
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            if (t + h * T < n) load(t + h * T, c[h]);
#pragma unroll
        for (int h = 0; h < kHold; ++h)
            if (t + h * T < n) {
                turn(c[h].u, c[h].w, c[h].a, turned, r[h]);
                most = most_of(r[h], most);
            }
    }
    for (int32_t i = t + kHold * T; i < n; i += T) {
        Chunk c;
        float x[8];
        load(i, c);
        turn(c.u, c.w, c.a, turned, x);
        most = most_of(x, most);
    }
    most = item_max<WAVES>(most, lds);
    const Scale s(most, it.lo > 0, before);
#pragma unroll
    for (int h = 0; h < kHold; ++h)
        if (t + h * T < n) store(t + h * T, r[h], s.inv);
    for (int32_t i = t + kHold * T; i < n; i += T) {
        Chunk c;
        float x[8];
        load(i, c);
        turn(c.u, c.w, c.a, turned, x);
        store(i, x, s.inv);
    }
    if (t == 0) *scale = s.s;
    if (!s.again) return;
    for (int32_t i = t * 16; i < it.lo * D; i += T * 16) {
        uint4 v = *reinterpret_cast<const uint4*>(y + i);
        v = make_uint4(codes_again(v.x, s.ratio), codes_again(v.y, s.ratio),
                       codes_again(v.z, s.ratio), codes_again(v.w, s.ratio));
        *reinterpret_cast<uint4*>(y + i) = v;
    }
}

// A lane takes two channels of 16 positions: 32 contiguous bytes of the cache.
template <int TYPE, bool VEC, int WAVES>
__device__ inline void value_item(const AppendArgs& p, const Item& it, uint32_t* lds)
{
    constexpr int T = 64 * WAVES;
    const int t = WAVES == 1 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
    const int32_t D = p.c.kv.D, half = D / 2;
    float* scale = p.c.v_scale + scale_at(p.c, it.pg, it.g, it.slot);
    const float before = it.lo > 0 ? *scale : 0.0f;
    int8_t* y = p.c.kv.v + (((it.pg * p.c.kv.G + it.g) << p.c.kv.shift) + it.slot) * D;
    const int32_t g0 = it.lo >> 4;  // first group of 16
    const int32_t n = (((it.hi + 15) >> 4) - g0) * half;
    struct Unit {
        uint32_t d[16][TYPE == MQ_F32 ? 2 : 1];
        __device__ float at(int j, int c) const
        {
            if constexpr (TYPE == MQ_F32) return __builtin_bit_cast(float, d[j][c]);
            else return half_of<TYPE>(d[j][0], c);
        }
    };
    // the unit's first token (from x0 on), its channel pair
    auto place = [&](int32_t i, int32_t& x, int32_t& d) {
        const int32_t g = div_by(i, p.inv_half);
        x = 16 * (g0 + g);
        d = 2 * (i - g * half);
    };
    auto load = [&](int32_t i, Unit& u) {
        int32_t x, d;
        place(i, x, d);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const bool in = x + j >= it.lo && x + j < it.hi;
            const int64_t at = (it.row + x + j) * p.ldv + (int64_t)it.g * D + d;
            if constexpr (TYPE == MQ_F32) {
                const uint32_t* v = static_cast<const uint32_t*>(p.v) + at;
                u.d[j][0] = in ? v[0] : 0;
                u.d[j][1] = in ? v[1] : 0;
            } else {
                const uint16_t* v = static_cast<const uint16_t*>(p.v) + at;
                if constexpr (VEC) u.d[j][0] = in ? *reinterpret_cast<const uint32_t*>(v) : 0;
                else u.d[j][0] = in ? v[0] | (uint32_t)v[1] << 16 : 0;
            }
        }
    };
    auto most_of = [](const Unit& u, uint32_t m) {
#pragma unroll
        for (int j = 0; j < 16; ++j) m = max(m, max(finite_bits(u.at(j, 0)), finite_bits(u.at(j, 1))));
        return m;
    };
    auto store = [&](int32_t i, const Unit& u, float inv) {
        int32_t x, d;
        place(i, x, d);
        int8_t* to = y + x * D + d * 16;
        if (x >= it.lo && x + 16 <= it.hi) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                uint32_t w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    w[j] = pack_codes(
                        block_code(u.at(4 * j, c), inv), block_code(u.at(4 * j + 1, c), inv),
                        block_code(u.at(4 * j + 2, c), inv), block_code(u.at(4 * j + 3, c), inv));
                *reinterpret_cast<uint4*>(to + 16 * c) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (x + j >= it.lo && x + j < it.hi) {
                    to[j] = (int8_t)block_code(u.at(j, 0), inv);
                    to[16 + j] = (int8_t)block_code(u.at(j, 1), inv);
                }
        }
    };
    Unit u;
    uint32_t most = 0;
    if (t < n) {
        load(t, u);
        most = most_of(u, most);
    }
    for (int32_t i = t + T; i < n; i += T) {
        Unit w;
        load(i, w);
        most = most_of(w, most);
    }
    most = item_max<WAVES>(most, lds);
    const Scale s(most, it.lo > 0, before);
    if (t < n) store(t, u, s.inv);
    for (int32_t i = t + T; i < n; i += T) {
        Unit w;
        load(i, w);
        store(i, w, s.inv);
    }
    if (t == 0) *scale = s.s;
    if (!s.again) return;
    // 16 tokens of a channel at a time; of the group that the new tokens begin
    // in only the bytes before them
    const int32_t old = it.lo;
    for (int32_t i = t; i < ((old + 15) >> 4) * D; i += T) {
        int8_t* at = y + (int64_t)i * 16;
        const int32_t first = div_by(i >> 1, p.inv_half) * 16;
        uint4 v = *reinterpret_cast<const uint4*>(at);
        v = make_uint4(codes_again(v.x, s.ratio), codes_again(v.y, s.ratio),
                       codes_again(v.z, s.ratio), codes_again(v.w, s.ratio));
        if (first + 16 <= old) {
            *reinterpret_cast<uint4*>(at) = v;
        } else {
            const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (first + j < old) at[j] = (int8_t)(w[j >> 2] >> (8 * (j & 3)));
        }
    }
}

// WAVES: of the four of a work-group that share an item.
template <int TYPE, bool VEC, int WAVES>
__global__ __launch_bounds__(256) void append_blocks_kernel(AppendArgs p)
{
    __shared__ uint32_t lds[4];
    const int64_t blk = blockIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (blk < p.rot) {
        rotate_queries<TYPE, VEC>(p, 4 * blk + wave);
        return;
    }
    const int64_t id = (blk - p.rot) * (4 / WAVES) + (WAVES == 1 ? wave : 0);
    Item it;
    if (id >= p.items || !find_item(p, id, it)) return;
    if (it.values) value_item<TYPE, VEC, WAVES>(p, it, lds);
    else key_item<TYPE, VEC, WAVES>(p, it, lds);
}

template <int TYPE, bool VEC>
hipError_t launch(AppendArgs& p, hipStream_t s)
{
    // a work-group per item where its elements fill more than a wave's chunks
    const int64_t B = p.c.kv.B, block = (int64_t)1 << p.c.bshift;
    const int64_t each = std::min(block, (p.T + B - 1) / B) * p.c.kv.D;
    const bool wide = each > 64 * 8 * kHold;
    const int64_t blocks = p.rot + (wide ? p.items : (p.items + 3) / 4);
    if (blocks >= kMaxBlocks) return hipErrorInvalidConfiguration;
    if (wide) append_blocks_kernel<TYPE, VEC, 4><<<(unsigned)blocks, 256, 0, s>>>(p);
    else append_blocks_kernel<TYPE, VEC, 1><<<(unsigned)blocks, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_t(AppendArgs& p, hipStream_t s)
{
    constexpr int E = TYPE == MQ_F32 ? 4 : 2;
    const auto ok = [](const void* x, int64_t ld) {
        return (uintptr_t)x % (4 * E) == 0 && ld % 4 == 0;
    };
    const bool vec = ok(p.q, p.ldq) && ok(p.k, p.ldk) && ok(p.v, p.ldv) && ok(p.q_out, p.ldo);
    return vec ? launch<TYPE, true>(p, s) : launch<TYPE, false>(p, s);
}

}  // namespace

hipError_t launch_append_blocks(const BlockCache& c, const void* q, int64_t ldq, const void* k,
                                int64_t ldk, const void* v, int64_t ldv, int32_t type, int64_t T,
                                int32_t H, const double* angles, int64_t positions, void* q_out,
                                int64_t ldo, hipStream_t s)
{
    AppendArgs p;
    p.c = c;
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
    const uint32_t per = (uint32_t)c.kv.D / 8, half = (uint32_t)c.kv.D / 2;
    p.per_turn = 64 / per;
    p.inv_per = (uint32_t)((((uint64_t)1 << 32) + per - 1) / per);
    p.inv_half = (uint32_t)((((uint64_t)1 << 32) + half - 1) / half);
    const int64_t turns = (H + p.per_turn - 1) / p.per_turn;
    p.waves = (int32_t)std::max<int64_t>(1, std::min<int64_t>(turns, 4096 / T));
    p.rot = (T * p.waves + 3) / 4;
    p.items = ((T >> c.bshift) + 2 * (int64_t)c.kv.B) * 2 * c.kv.G;
    if (p.items >= 4 * kMaxBlocks) return hipErrorInvalidConfiguration;
    if (type == MQ_F32) return launch_t<MQ_F32>(p, s);
    return type == MQ_BF16 ? launch_t<MQ_BF16>(p, s) : launch_t<MQ_F16>(p, s);
}

}  // namespace mq
