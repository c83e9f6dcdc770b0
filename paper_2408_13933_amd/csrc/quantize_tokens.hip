// Token quantizer: every row's codes by its own largest magnitude.
//
// A row stays in registers between its maximum and its codes, so it is read
// once; rows of more than 16384 elements are read again (from the L2).  Memory
// bounds it at many tokens, a round trip to memory, the reduction and the store
// at few: 2048 rows of 2048 fp16 numbers 5.4 us (2.3 TB/s of reads and codes, a launch
// of one round), 16 of 5632 bf16 ones 3.0.
#include <algorithm>

#include "linear_tokens.h"
#include "wave.h"

namespace mq {
namespace {

constexpr int kVec = 8;  // elements of a lane's chunk

struct QuantArgs {
    const void* x;
    int8_t* x_q;
    float* scale;
    int32_t* rowsum;  // or nullptr
    int32_t* clear;   // counters that a K split of the product needs at 0
    int64_t clear_n;
    int64_t M, K, ldx;
};

// The larger of the waves' values (WAVES of 4 share a row).
template <int WAVES>
__device__ inline uint32_t row_max(uint32_t v, uint32_t* lds)
{
    v = wave_max(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = max(max(lds[0], lds[1]), max(lds[2], lds[3]));
    }
    return v;
}
template <int WAVES>
__device__ inline int32_t row_sum(int32_t v, int32_t* lds)
{
    v = (int32_t)wave_sum(v);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0] + lds[1] + lds[2] + lds[3];
    }
    return v;
}

template <int TYPE>
__device__ inline uint32_t chunk_max(const Raw<TYPE, kVec>& r)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) m = max(m, abs_bits(r[i]));
    return m;
}
template <int TYPE>
__device__ inline uint2 chunk_codes(const Raw<TYPE, kVec>& r, float inv, bool bad)
{
    uint32_t c[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) c[i] = code_bits(r[i], inv);
    uint2 v = make_uint2(pack_codes(c[0], c[1], c[2], c[3]), pack_codes(c[4], c[5], c[6], c[7]));
    if (bad) v = make_uint2(0, 0);
    return v;
}

// CH chunks of a lane held in registers, 0: the row is walked over twice.
// VEC: whole 16-byte accesses; else single elements.
template <int TYPE, int WAVES, int CH, bool VEC>
__global__ __launch_bounds__(256) void quantize_tokens_kernel(QuantArgs p)
{
    __shared__ uint32_t lds[2][4];
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.clear_n;
         i += (int64_t)gridDim.x * 256)
        p.clear[i] = 0;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t m = (int64_t)blockIdx.x * (4 / WAVES) + (WAVES == 1 ? wave : 0);
    if (m >= p.M) return;  // whole waves, whole blocks where they share a row
    const int t = WAVES == 1 ? (int)threadIdx.x & 63 : (int)threadIdx.x;
    constexpr int T = 64 * WAVES;
    constexpr int E = TYPE == MQ_F32 ? 4 : 2;
    const int8_t* x = static_cast<const int8_t*>(p.x) + m * p.ldx * E;
    int8_t* y = p.x_q + m * p.K;
    const int K = (int)p.K;
    uint32_t most = 0;
    int32_t sum = 0;
    Raw<TYPE, kVec> r[CH ? CH : 1];
    if constexpr (!VEC) {
        for (int k = t; k < K; k += T) most = max(most, abs_bits(load_elem<TYPE>(x, k)));
    } else if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * T + t) * kVec;
            if (k < K) r[c].load(x + k * E);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if ((c * T + t) * kVec < K) most = max(most, chunk_max<TYPE>(r[c]));
    } else {
        for (int k = t * kVec; k < K; k += T * kVec) {
            r[0].load(x + k * E);
            most = max(most, chunk_max<TYPE>(r[0]));
        }
    }
    most = row_max<WAVES>(most, lds[0]);
    const bool bad = most >= kInfBits;
    const float scale = scale_of(most), inv = 1.0f / scale;
    if (t == 0) p.scale[m] = bad ? __builtin_nanf("") : scale;
    auto put = [&](int k, const Raw<TYPE, kVec>& v) {
        const uint2 c = chunk_codes<TYPE>(v, inv, bad);
        *reinterpret_cast<uint2*>(y + k) = c;
        sum = __builtin_amdgcn_sdot4((int)c.x, 0x01010101, sum, false);
        sum = __builtin_amdgcn_sdot4((int)c.y, 0x01010101, sum, false);
    };
    if constexpr (!VEC) {
        for (int k = t; k < K; k += T) {
            const int8_t c = bad ? 0 : (int8_t)code_bits(load_elem<TYPE>(x, k), inv);
            y[k] = c;
            sum += c;
        }
    } else if constexpr (CH > 0) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int k = (c * T + t) * kVec;
            if (k < K) put(k, r[c]);
        }
    } else {
        for (int k = t * kVec; k < K; k += T * kVec) {
            r[0].load(x + k * E);
            put(k, r[0]);
        }
    }
    if (p.rowsum) {
        sum = row_sum<WAVES>(sum, reinterpret_cast<int32_t*>(lds[1]));
        if (t == 0) p.rowsum[m] = sum;
    }
}

template <int TYPE, int WAVES, int CH, bool VEC>
hipError_t launch(const QuantArgs& p, hipStream_t s)
{
    const int64_t rows = 4 / WAVES;
    quantize_tokens_kernel<TYPE, WAVES, CH, VEC>
        <<<(unsigned)((p.M + rows - 1) / rows), 256, 0, s>>>(p);
    return hipGetLastError();
}

template <int TYPE>
hipError_t launch_t(const QuantArgs& p, hipStream_t s)
{
    constexpr int E = TYPE == MQ_F32 ? 4 : 2;
    const bool vec = p.K % kVec == 0 && (uintptr_t)p.x % 16 == 0 && (p.ldx * E) % 16 == 0 &&
                     (uintptr_t)p.x_q % 8 == 0;
    if (!vec) return launch<TYPE, 4, 0, false>(p, s);
    // a wave per row of one chunk per lane, else four waves
    if (p.K <= 64 * kVec) return launch<TYPE, 1, 1, true>(p, s);
    if (p.K <= 256 * kVec) return launch<TYPE, 4, 1, true>(p, s);
    if (p.K <= 256 * kVec * 2) return launch<TYPE, 4, 2, true>(p, s);
    if (p.K <= 256 * kVec * 4) return launch<TYPE, 4, 4, true>(p, s);
    if (p.K <= 256 * kVec * 8) return launch<TYPE, 4, 8, true>(p, s);
    return launch<TYPE, 4, 0, true>(p, s);
}

}  // namespace

hipError_t launch_quantize_tokens(const void* x, int32_t type, int64_t M, int64_t K, int64_t ldx,
                                  int8_t* x_q, float* scale, int32_t* rowsum, int32_t* clear,
                                  int64_t clear_n, hipStream_t s)
{
    const QuantArgs p{x, x_q, scale, rowsum, clear, clear_n, M, K, ldx};
    if (type == MQ_F32) return launch_t<MQ_F32>(p, s);
    return type == MQ_BF16 ? launch_t<MQ_BF16>(p, s) : launch_t<MQ_F16>(p, s);
}

}  // namespace mq
