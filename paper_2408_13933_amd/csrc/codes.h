// Requantization of fp64 values to activation codes and the 8-code loads and
// stores, shared by the kernels that evaluate an operator in fp64 and write
// codes (the decoder-block glue, the rotation into the key/value cache).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mq {

// The code before its clamp to the output range: rint(t) + zy.  A quotient
// beyond +-2^17 saturates whatever the zero-point (|zy| <= 2^15), so it is
// limited there first (NaN: the low end) and adding 1.5 * 2^52 leaves rint(t)
// (to nearest, ties to even) in the low word: 32-bit integers throughout.
__device__ inline double limit_quotient(double t)
{
    return fmin(fmax(t, -131072.0), 131072.0);
}
constexpr double kRintShift = 6755399441055744.0;  // 1.5 * 2^52
__device__ inline int32_t rint_low(double shifted)
{
    return (int32_t)(uint32_t)__double_as_longlong(shifted);
}

// 2^x for -2^30 < x < 1024 (to 0 far below -1022): rint by the 1.5 * 2^52 shift, a
// polynomial of degree 10 through the Chebyshev nodes of [-1/2, 1/2] (within
// 3e-16 of 2^f), the exponent added.
__device__ inline double exp2_poly(double x)
{
    const double t = x + kRintShift;
    const double f = x - (t - kRintShift);
    double p = 0x1.e6063f7217bc6p-28;
    p = __builtin_fma(p, f, 0x1.b675bca4eeebbp-24);
    p = __builtin_fma(p, f, 0x1.62bfd47773353p-20);
    p = __builtin_fma(p, f, 0x1.ffcb54062e698p-17);
    p = __builtin_fma(p, f, 0x1.430913096fd9fp-13);
    p = __builtin_fma(p, f, 0x1.5d87fe9d7a584p-10);
    p = __builtin_fma(p, f, 0x1.3b2ab6fba1ddap-7);
    p = __builtin_fma(p, f, 0x1.c6b08d703ce49p-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff82c598p-3);
    p = __builtin_fma(p, f, 0x1.62e42fefa3a19p-1);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, rint_low(t));
}

// The same by a table of 2^(j/64): adding kTableShift leaves 64 x, rounded, in
// the low word, and the rest, |f| <= 1/128, takes a polynomial of degree 4
// (within 2.5e-15 of 2^f).
constexpr double kTableShift = 105553116266496.0;  // 1.5 * 2^46
__device__ inline double exp2_rest(double f)
{
    double p = 0x1.3b2ad0385b409p-7;
    p = __builtin_fma(p, f, 0x1.c6b0c40d8c4e9p-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff82ac52p-3);
    p = __builtin_fma(p, f, 0x1.62e42fefa0352p-1);
    return __builtin_fma(p, f, 1.0);
}

template <int BITS>
__device__ inline int32_t clamp_code(int32_t q)
{
    constexpr int32_t qmin = -(1 << (BITS - 1)), qmax = (1 << (BITS - 1)) - 1;
    return min(max(q, qmin), qmax);
}

template <int BITS>
__device__ inline int32_t requant_f64(double v, double ay, int32_t zy)
{
#pragma clang fp contract(off)
    return clamp_code<BITS>(rint_low(limit_quotient(v / ay) + kRintShift) + zy);
}

// N codes.  exact(u) is the quotient of code u as the definition evaluates it
// (its divisions correctly rounded), fast(u) the same quotient through
// products with reciprocals: for RMSNorm six roundings against three, within
// 2^-49 of it relatively.  For |t| <= 2^17 that is within 2^-32, so where
// fast(u) is further than 2^-30 from every half-integer both round to the same
// integer; a wave with a code nearer than that evaluates exact(u) for all of
// its codes.  These kernels are
// bound by the vector ALU at prompt sizes: with the division, 64-bit integer
// conversions and clamps per code, RMSNorm of 1024 x 2048 took 9.4 us
// instead of 4.7, with the residual add 10.9 instead of 6.8, the gated
// product of 1024 x 5632 12.0 instead of 8.3.
template <int BITS, int N, class Exact, class Fast>
__device__ inline void requant_codes(int32_t* q, int32_t zy, Exact exact, Fast fast)
{
#pragma clang fp contract(off)
    double far = 0.0;
#pragma unroll
    for (int u = 0; u < N; ++u) {
        const double t = limit_quotient(fast(u));
        const double r = t + kRintShift;
        q[u] = clamp_code<BITS>(rint_low(r) + zy);
        far = fmax(far, fabs(t - (r - kRintShift)));
    }
    if (__builtin_expect(__ballot(far > 0.5 - 0x1p-30) != 0, 0)) {
#pragma unroll
        for (int u = 0; u < N; ++u)
            q[u] = clamp_code<BITS>(rint_low(limit_quotient(exact(u)) + kRintShift) + zy);
    }
}

template <int BITS>
__device__ inline void store_code(void* y, int64_t i, int32_t v)
{
    if constexpr (BITS == 8) static_cast<int8_t*>(y)[i] = (int8_t)v;
    else static_cast<int16_t*>(y)[i] = (int16_t)v;
}

// Eight codes to y[i .. i+7] with one 8-byte (int8) or 16-byte (int16)
// store; i is a multiple of 8 and y is 16-byte aligned.
template <int BITS>
__device__ inline void store8(void* y, int64_t i, const int32_t* q)
{
    if constexpr (BITS == 8) {
        uint2 o;
        o.x = ((uint32_t)(uint8_t)q[0]) | ((uint32_t)(uint8_t)q[1] << 8) |
              ((uint32_t)(uint8_t)q[2] << 16) | ((uint32_t)(uint8_t)q[3] << 24);
        o.y = ((uint32_t)(uint8_t)q[4]) | ((uint32_t)(uint8_t)q[5] << 8) |
              ((uint32_t)(uint8_t)q[6] << 16) | ((uint32_t)(uint8_t)q[7] << 24);
        *reinterpret_cast<uint2*>(static_cast<int8_t*>(y) + i) = o;
    } else {
        int4 o;
        o.x = (int)(((uint32_t)(uint16_t)q[0]) | ((uint32_t)(uint16_t)q[1] << 16));
        o.y = (int)(((uint32_t)(uint16_t)q[2]) | ((uint32_t)(uint16_t)q[3] << 16));
        o.z = (int)(((uint32_t)(uint16_t)q[4]) | ((uint32_t)(uint16_t)q[5] << 16));
        o.w = (int)(((uint32_t)(uint16_t)q[6]) | ((uint32_t)(uint16_t)q[7] << 16));
        *reinterpret_cast<int4*>(static_cast<int16_t*>(y) + i) = o;
    }
}

// The eight int16 codes of one 16-byte load.
typedef int v4i __attribute__((ext_vector_type(4)));
__device__ inline void unpack8(const v4i v, int32_t* c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        c[2 * i] = (int32_t)(int16_t)v[i];
        c[2 * i + 1] = v[i] >> 16;
    }
}

}  // namespace mq
