// Penalties for words that a sequence holds, biases and grammar masks, on logits
// where they lie.
//
// A work-group takes a row's range of kWords words: it walks over the row's whole
// history and counts the words of its range in LDS, so that order does not matter
// and a word's penalties, bias and mask meet in one thread.  Only words that
// change are read or written.  Latency bounds it for few rows (row lengths, the
// history, the logits: three round trips), the history and the -infinities that
// masks write for many.
#include <algorithm>

#include "adjust.h"
#include "kvcache.h"
#include "tokens.h"

namespace mq {
namespace {

constexpr int kThreads = 512;
constexpr int kEach = 8;  // consecutive words of a thread
constexpr int kWords = kThreads * kEach;

// A word's entry: how often the sequence holds it past its prompt, and kPrompt if
// the prompt does.
constexpr uint32_t kPrompt = 0x80000000u;

template <int TYPE>
__device__ inline void store_bits(void* x, int64_t i, uint32_t b)
{
    if constexpr (TYPE == MQ_F32) static_cast<uint32_t*>(x)[i] = b;
    else static_cast<uint16_t*>(x)[i] = (uint16_t)b;
}
template <int TYPE>
constexpr uint32_t kMinusInf = TYPE == MQ_F32 ? 0xff800000u : TYPE == MQ_BF16 ? 0xff80u : 0xfc00u;

template <int TYPE, bool BIAS>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs p, int32_t ranges, bool vec_x,
                                                          bool vec_h)
{
#pragma clang fp contract(off)
    __shared__ __attribute__((aligned(16))) uint32_t count[kWords];
    __shared__ __attribute__((aligned(16))) uint32_t entry[BIAS ? kWords : 4];  // of the bias list, + 1
    const int tid = threadIdx.x;
    const int64_t m = blockIdx.x / ranges;
    const int32_t w0 = (int32_t)(blockIdx.x - m * ranges) * kWords;
    const int32_t V = (int32_t)p.V, first = w0 + tid * kEach;
    const int32_t words = min(kWords, V - w0);

    // the mask's byte of this thread's words (words past the row: allowed)
    uint32_t allowed = 0xff;
    if (p.mask && first < V) {
        allowed = (p.mask[m * p.ldm + (first >> 5)] >> (first & 31)) & 0xff;
        if (first + kEach > V) allowed |= 0xff << (V - first);
    }
    const float rep = p.repetition ? p.repetition[m] : 1.0f;
    const float pres = p.presence ? p.presence[m] : 0.0f;
    const float freq = p.frequency ? p.frequency[m] : 0.0f;
    // (x / 1, x - 0 and x - 0 * n change no bit)
    const bool penal = p.history && !(rep == 1.0f && pres == 0.0f && freq == 0.0f);
    int32_t b0 = 0, b1 = 0;
    if constexpr (BIAS) {
        b0 = max(p.bias_starts[m], 0);
        b1 = (int32_t)min((int64_t)p.bias_starts[m + 1], p.bias_n);
    }
    if (penal || b0 < b1) {
        const uint4 zero = make_uint4(0, 0, 0, 0);
        for (int i = tid; i < kWords / 4; i += kThreads) {
            reinterpret_cast<uint4*>(count)[i] = zero;
            if constexpr (BIAS) reinterpret_cast<uint4*>(entry)[i] = zero;
        }
        __syncthreads();
    }
    if (penal) {
        const int32_t n = (int32_t)min((int64_t)p.hist_lens[m], p.cols);
        const int32_t prompt = p.prompt_lens ? p.prompt_lens[m] : 0;
        const int32_t* h = p.history + m * p.ldh;
        auto add = [&](int32_t i, int32_t word) {
            const uint32_t at = (uint32_t)word - (uint32_t)w0;
            if (at >= (uint32_t)words) return;
            if (i < prompt) atomicOr(&count[at], kPrompt);
            else atomicAdd(&count[at], 1u);
        };
        if (vec_h) {
            for (int32_t i = tid * 4; i < n; i += kThreads * 4) {
                const int4 v = *reinterpret_cast<const int4*>(h + i);  // (whole fours of a row)
                add(i, v.x);
                if (i + 1 < n) add(i + 1, v.y);
                if (i + 2 < n) add(i + 2, v.z);
                if (i + 3 < n) add(i + 3, v.w);
            }
        } else {
            for (int32_t i = tid; i < n; i += kThreads) add(i, h[i]);
        }
    }
    if constexpr (BIAS) {
        for (int32_t i = b0 + tid; i < b1; i += kThreads) {
            const uint32_t at = (uint32_t)p.bias_tokens[i] - (uint32_t)w0;
            // of equal words the last one
            if (at < (uint32_t)words) atomicMax(&entry[at], (uint32_t)i + 1);
        }
    }
    uint32_t c[kEach] = {}, e[kEach] = {}, touched = 0;
    if (penal || b0 < b1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            c[i] = count[tid * kEach + i];
            if constexpr (BIAS) e[i] = entry[tid * kEach + i];
            if (c[i] | e[i]) touched |= 1u << i;
        }
    }
    if (first >= V) return;
    touched &= allowed;
    if (touched == 0 && allowed == 0xff) return;
    const int64_t at = m * p.ld + first;
    auto value = [&](int i, float x) {
        if (c[i]) {
            x = x > 0.0f ? x / rep : x * rep;
            if (const uint32_t n = c[i] & ~kPrompt) {
                x = x - freq * (float)n;
                x = x - pres;
            }
        }
        if (BIAS && e[i]) x = x + p.bias_values[e[i] - 1];
        return x;
    };
    if (allowed == 0 && vec_x && first + kEach <= V) {
        constexpr uint32_t b = TYPE == MQ_F32 ? kMinusInf<TYPE> : kMinusInf<TYPE> * 0x10001u;
        uint4* y = reinterpret_cast<uint4*>(static_cast<int8_t*>(p.x) + at * (TYPE == MQ_F32 ? 4 : 2));
        y[0] = make_uint4(b, b, b, b);
        if constexpr (TYPE == MQ_F32) y[1] = make_uint4(b, b, b, b);
        return;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (!((allowed >> i) & 1)) store_bits<TYPE>(p.x, at + i, kMinusInf<TYPE>);
        else if ((touched >> i) & 1)
            store_elem<TYPE>(p.x, at + i, value(i, load_elem<TYPE>(p.x, at + i)));
    }
}

template <int TYPE>
hipError_t launch(const AdjustArgs& p, hipStream_t s)
{
    const int64_t ranges = (p.V + kWords - 1) / kWords;
    if (p.M * ranges >= kMaxBlocks / 2) return hipErrorInvalidConfiguration;  // of 512 threads
    const bool vec_x = (uintptr_t)p.x % 16 == 0 && p.ld * type_bytes(TYPE) % 16 == 0;
    const bool vec_h = (uintptr_t)p.history % 16 == 0 && p.ldh % 4 == 0 && p.cols % 4 == 0;
    const unsigned n = (unsigned)(p.M * ranges);
    if (p.bias_starts) adjust_kernel<TYPE, true><<<n, kThreads, 0, s>>>(p, (int32_t)ranges, vec_x, vec_h);
    else adjust_kernel<TYPE, false><<<n, kThreads, 0, s>>>(p, (int32_t)ranges, vec_x, vec_h);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& p, int32_t type, hipStream_t s)
{
    if (type == MQ_F32) return launch<MQ_F32>(p, s);
    return type == MQ_BF16 ? launch<MQ_BF16>(p, s) : launch<MQ_F16>(p, s);
}

}  // namespace mq
