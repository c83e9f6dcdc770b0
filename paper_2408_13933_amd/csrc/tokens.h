// Floating-point elements (fp32, bf16, fp16) of the operators whose scales are
// found at run time: conversions, the scale of a largest magnitude and the
// codes by it, the output of a product with a scale per token.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "mq.h"

namespace mq {

// What a product with activation scales per token has besides QLinearArgs.
struct TokenArgs {
    const float* scale;  // [M]
    void* y;             // [M][N]
    int32_t type;        // of y
};

__host__ __device__ inline bool type_ok(int32_t t) { return t >= MQ_F32 && t <= MQ_F16; }
__host__ __device__ inline int type_bytes(int32_t t) { return t == MQ_F32 ? 4 : 2; }

typedef float tok_v2f __attribute__((ext_vector_type(2)));
typedef __bf16 tok_v2b __attribute__((ext_vector_type(2)));
typedef _Float16 tok_v2h __attribute__((ext_vector_type(2)));

// Two values in one dword, the first in the low half, each rounded to nearest
// even.
template <int TYPE>
__device__ inline uint32_t pack2(float a, float b)
{
    const tok_v2f v = {a, b};
    if constexpr (TYPE == MQ_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, tok_v2b));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, tok_v2h));
}

// The half of a dword of 2-byte elements as fp32 (exact).
template <int TYPE>
__device__ inline float half_of(uint32_t d, int high)
{
    if constexpr (TYPE == MQ_BF16)
        return __builtin_bit_cast(float, high ? d & 0xffff0000u : d << 16);
    else
        return (float)__builtin_bit_cast(tok_v2h, d)[high];
}

template <int TYPE>
__device__ inline float load_elem(const void* x, int64_t i)
{
    if constexpr (TYPE == MQ_F32) return static_cast<const float*>(x)[i];
    else return half_of<TYPE>(static_cast<const uint16_t*>(x)[i], 0);
}
template <int TYPE>
__device__ inline void store_elem(void* y, int64_t i, float v)
{
    if constexpr (TYPE == MQ_F32) static_cast<float*>(y)[i] = v;
    else static_cast<uint16_t*>(y)[i] = (uint16_t)pack2<TYPE>(v, 0.0f);
}

// N consecutive elements as they lie in memory, in dwords; 16-byte accesses.
template <int TYPE, int N>
struct Raw {
    static constexpr int kDwords = N * (TYPE == MQ_F32 ? 4 : 2) / 4;
    uint32_t d[kDwords];
    __device__ void load(const void* x)
    {
#pragma unroll
        for (int i = 0; i < kDwords / 4; ++i) {
            const uint4 v = static_cast<const uint4*>(x)[i];
            d[4 * i] = v.x;
            d[4 * i + 1] = v.y;
            d[4 * i + 2] = v.z;
            d[4 * i + 3] = v.w;
        }
    }
    __device__ float operator[](int i) const
    {
        if constexpr (TYPE == MQ_F32) return __builtin_bit_cast(float, d[i]);
        else return half_of<TYPE>(d[i >> 1], i & 1);
    }
};

// Magnitudes compare as their bits do; NaN is above infinity, both at and
// above kInfBits.
constexpr uint32_t kInfBits = 0x7f800000u;
__device__ inline uint32_t abs_bits(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

// The scale of 8-bit codes for a largest magnitude, max(a, 2^-60) / 127: the
// floor keeps 1 / scale (and, in the attention, sums of weights over value
// scales) far from overflow.
constexpr float kTinyAbs = 0x1p-60f;
__device__ inline float scale_of(uint32_t abs)
{
    return fmaxf(__builtin_bit_cast(float, abs), kTinyAbs) / 127.0f;
}

// The code of x by inv = 1 / scale, rint(x inv), in the low byte: adding 1.5 * 2^23
// rounds as rint does and leaves the integer in the low bits.  |x| <= 127 scale
// (1 + 2^-24), so the product is below 127.0001 and needs no clamp.
__device__ inline uint32_t code_bits(float x, float inv)
{
    return __builtin_bit_cast(uint32_t, x * inv + 12582912.0f);
}
__device__ inline uint32_t pack_codes(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x04000c0cu);
    return lo | hi;
}

// An output of the token product from its exact integer sum.
__device__ inline float token_output(int32_t c, float w_scale, float a_scale, float bias)
{
#pragma clang fp contract(off)
    const float t = (float)c * w_scale;
    return t * a_scale + bias;
}

}  // namespace mq
