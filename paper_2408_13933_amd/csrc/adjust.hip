// Penalties for words that a sequence holds, biases and grammar masks, on logits
// where they lie.
//
// A work-group takes a row's range of words: it walks over the row's whole history
// and counts the words of its range in LDS, so that order does not matter and a
// word's penalties, bias and mask meet in one thread.  Only groups of eight words
// with one that changes are read or written.  Latency bounds it: row lengths and the
// history's first 2048 words in one round trip, a trip for each of the words that a thread
// counts past them, then bias values and logits: one row of 256000 fp32 words, 9000 of
// history and 300 biases 7.1 us, 200 rows of 32000 bf16 ones with 1500 of history and
// masks 13.8 (8 MB).
#include <algorithm>

#include "adjust.h"
#include "kvcache.h"
#include "tokens.h"

namespace mq {
namespace {

constexpr int kThreads = 512;

// A word's state in LDS.  Packed: an entry of the bias list + 1 in the upper bits, then
// whether the prompt holds the word, then how often the sequence does past its prompt;
// 8192 words are a work-group's, so that 200 rows of 32000 fit the chip at once.  Else
// two numbers of 32 bits, 4096 words.
template <bool PACKED, int EACH>
struct State {
    static constexpr int kWords = kThreads * EACH;  // consecutive ones of a thread
    static constexpr int kEntry = PACKED ? 15 : 0;  // its lowest bit
    static constexpr uint32_t kPrompt = PACKED ? 1u << 14 : 1u << 31;
    __attribute__((aligned(16))) uint32_t count[kWords];
    __attribute__((aligned(16))) uint32_t own[PACKED ? 4 : kWords];
    __device__ uint32_t* entry() { return PACKED ? count : own; }
};
constexpr int64_t kPackedCols = (1 << 14) - 1, kPackedBias = (1 << 17) - 2;

template <int TYPE>
constexpr uint32_t kMinusInf = TYPE == MQ_F32 ? 0xff800000u : TYPE == MQ_BF16 ? 0xff80u : 0xfc00u;

// Eight logits as they lie in memory.
template <int TYPE>
struct Eight {
    static constexpr int kDwords = TYPE == MQ_F32 ? 8 : 4;
    uint32_t d[kDwords];
    __device__ void load(const void* x, int64_t i)
    {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const int8_t*>(x) +
                                                        i * (TYPE == MQ_F32 ? 4 : 2));
#pragma unroll
        for (int j = 0; j < kDwords / 4; ++j) {
            const uint4 v = p[j];
            d[4 * j] = v.x, d[4 * j + 1] = v.y, d[4 * j + 2] = v.z, d[4 * j + 3] = v.w;
        }
    }
    __device__ void store(void* x, int64_t i) const
    {
        uint4* p =
            reinterpret_cast<uint4*>(static_cast<int8_t*>(x) + i * (TYPE == MQ_F32 ? 4 : 2));
#pragma unroll
        for (int j = 0; j < kDwords / 4; ++j)
            p[j] = make_uint4(d[4 * j], d[4 * j + 1], d[4 * j + 2], d[4 * j + 3]);
    }
    __device__ float get(int i) const
    {
        if constexpr (TYPE == MQ_F32) return __builtin_bit_cast(float, d[i]);
        else return half_of<TYPE>(d[i >> 1], i & 1);
    }
    __device__ void put(int i, uint32_t b)
    {
        if constexpr (TYPE == MQ_F32) d[i] = b;
        else d[i >> 1] = (i & 1) ? (d[i >> 1] & 0xffffu) | b << 16 : (d[i >> 1] & 0xffff0000u) | b;
    }
};
template <int TYPE>
__device__ inline uint32_t bits_of(float x)
{
    if constexpr (TYPE == MQ_F32) return __builtin_bit_cast(uint32_t, x);
    else return pack2<TYPE>(x, 0.0f) & 0xffffu;
}
template <int TYPE>
__device__ inline void store_bits(void* x, int64_t i, uint32_t b)
{
    if constexpr (TYPE == MQ_F32) static_cast<uint32_t*>(x)[i] = b;
    else static_cast<uint16_t*>(x)[i] = (uint16_t)b;
}

template <int TYPE, bool PACKED, int kEach>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs p, int32_t ranges, bool vec_x,
                                                          bool vec_h)
{
#pragma clang fp contract(off)
    using S = State<PACKED, kEach>;
    constexpr int kWords = S::kWords;
    __shared__ S st;
    const int tid = threadIdx.x;
    const int64_t m = blockIdx.x / ranges;
    const int32_t w0 = (int32_t)(blockIdx.x - m * ranges) * kWords;
    const int32_t V = (int32_t)p.V, first = w0 + tid * kEach;
    const int32_t words = min(kWords, V - w0);

    // everything that depends on the row alone, the first words of its history too (they
    // are there up to `cols`, counted or not)
    int32_t n = 0, prompt = 0;
    const int32_t* h = nullptr;
    int4 ahead = make_int4(0, 0, 0, 0);
    if (p.history) {
        n = (int32_t)min((int64_t)p.hist_lens[m], p.cols);
        prompt = p.prompt_lens ? p.prompt_lens[m] : 0;
        h = p.history + m * p.ldh;
        if (vec_h && tid * 4 < p.cols) ahead = reinterpret_cast<const int4*>(h)[tid];
    }
    const float rep = p.repetition ? p.repetition[m] : 1.0f;
    const float pres = p.presence ? p.presence[m] : 0.0f;
    const float freq = p.frequency ? p.frequency[m] : 0.0f;
    // (unsigned: what threads add to them stays below 2^32)
    uint32_t b0 = 0, b1 = 0;
    if (p.bias_starts) {
        b1 = (uint32_t)min((int64_t)max(p.bias_starts[m + 1], 0), p.bias_n);
        b0 = min((uint32_t)max(p.bias_starts[m], 0), b1);
    }
    // the mask's bits of this thread's words (words past the row: allowed)
    constexpr uint32_t kAll = (1u << kEach) - 1;
    uint32_t allowed = kAll;
    if (p.mask && first < V) {
        allowed = (p.mask[m * p.ldm + (first >> 5)] >> (first & 31)) & kAll;
        if (first + kEach > V) allowed |= kAll & (kAll << (V - first));
    }
    // (x / 1, x - 0 and x - 0 * n change no bit)
    const bool penal = n > 0 && !(rep == 1.0f && pres == 0.0f && freq == 0.0f);
    uint32_t c[kEach] = {}, e[kEach] = {}, touched = 0;
    if (penal || b0 < b1) {
        int32_t word = b0 + tid < b1 ? p.bias_tokens[b0 + tid] : -1;
        const uint4 zero = make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kEach / 4; ++i) {
            reinterpret_cast<uint4*>(st.count)[i * kThreads + tid] = zero;
            if constexpr (!PACKED) reinterpret_cast<uint4*>(st.own)[i * kThreads + tid] = zero;
        }
        __syncthreads();
        for (uint32_t i = b0 + tid; i < b1; i += kThreads) {
            if (i != b0 + tid) word = p.bias_tokens[i];
            const uint32_t at = (uint32_t)word - (uint32_t)w0;
            // of equal words the last one
            if (at < (uint32_t)words) atomicMax(&st.entry()[at], (i + 1) << S::kEntry);
        }
        if (PACKED && b0 < b1) __syncthreads();  // (the maxima are of entries alone)
        if (penal) {
            auto add = [&](uint32_t i, int32_t word) {
                const uint32_t at = (uint32_t)word - (uint32_t)w0;
                if (i >= (uint32_t)n || at >= (uint32_t)words) return;
                if ((int32_t)i < prompt) atomicOr(&st.count[at], S::kPrompt);
                else atomicAdd(&st.count[at], 1u);
            };
            auto add_four = [&](uint32_t i, const int4& v) {
                add(i, v.x);
                add(i + 1, v.y);
                add(i + 2, v.z);
                add(i + 3, v.w);
            };
            if (vec_h) {
                add_four(tid * 4, ahead);
                for (uint32_t i = (kThreads + tid) * 4; i < (uint32_t)n; i += kThreads * 4)
                    add_four(i, *reinterpret_cast<const int4*>(h + i));  // (read word by word)
            } else {
                for (uint32_t i = tid; i < (uint32_t)n; i += kThreads) add(i, h[i]);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            c[i] = st.count[tid * kEach + i];
            if constexpr (PACKED) {
                e[i] = c[i] >> S::kEntry;
                c[i] &= (1u << S::kEntry) - 1;
            } else {
                e[i] = st.own[tid * kEach + i];
            }
            if (c[i] | e[i]) touched |= 1u << i;
        }
    }
    if (first >= V) return;
    touched &= allowed;
    if (touched == 0 && allowed == kAll) return;
    const int64_t at = m * p.ld + first;
    float bias[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        bias[i] = 0.0f;
        if (e[i] && ((touched >> i) & 1)) bias[i] = p.bias_values[e[i] - 1];
    }
    auto value = [&](int i, float x) {
        if (c[i]) {
            x = x > 0.0f ? x / rep : x * rep;
            if (const uint32_t k = c[i] & ~S::kPrompt) {
                x = x - freq * (float)k;
                x = x - pres;
            }
        }
        if (e[i]) x = x + bias[i];
        return x;
    };
    if (vec_x && first + kEach <= V) {
        Eight<TYPE> x[kEach / 8];
#pragma unroll
        for (int j = 0; j < kEach / 8; ++j)
            if (((touched >> (8 * j)) & 0xff) != 0 ||
                (((allowed >> (8 * j)) & 0xff) != 0xff && ((allowed >> (8 * j)) & 0xff) != 0))
                x[j].load(p.x, at + 8 * j);
#pragma unroll
        for (int j = 0; j < kEach / 8; ++j) {
            const uint32_t ok = (allowed >> (8 * j)) & 0xff, to = (touched >> (8 * j)) & 0xff;
            if (to == 0 && ok == 0xff) continue;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (!((ok >> i) & 1)) x[j].put(i, kMinusInf<TYPE>);
                else if ((to >> i) & 1) x[j].put(i, bits_of<TYPE>(value(8 * j + i, x[j].get(i))));
            }
            x[j].store(p.x, at + 8 * j);
        }
        return;
    }
    float x[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) x[i] = (touched >> i) & 1 ? load_elem<TYPE>(p.x, at + i) : 0.0f;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        if (!((allowed >> i) & 1)) store_bits<TYPE>(p.x, at + i, kMinusInf<TYPE>);
        else if ((touched >> i) & 1) store_bits<TYPE>(p.x, at + i, bits_of<TYPE>(value(i, x[i])));
    }
}

template <int TYPE, bool PACKED, int EACH>
hipError_t launch_p(const AdjustArgs& p, hipStream_t s)
{
    constexpr int kWords = State<PACKED, EACH>::kWords;
    const int64_t ranges = (p.V + kWords - 1) / kWords;
    if (p.M * ranges >= kMaxBlocks / 2) return hipErrorInvalidConfiguration;  // of 512 threads
    const bool vec_x = (uintptr_t)p.x % 16 == 0 && p.ld * type_bytes(TYPE) % 16 == 0;
    const bool vec_h = (uintptr_t)p.history % 16 == 0 && p.ldh % 4 == 0 && p.cols % 4 == 0;
    adjust_kernel<TYPE, PACKED, EACH>
        <<<(unsigned)(p.M * ranges), kThreads, 0, s>>>(p, (int32_t)ranges, vec_x, vec_h);
    return hipGetLastError();
}
template <int TYPE>
hipError_t launch(const AdjustArgs& p, hipStream_t s)
{
    const bool fits = (!p.history || p.cols <= kPackedCols) &&
                      (!p.bias_starts || p.bias_n <= kPackedBias);
    if (!fits) return launch_p<TYPE, false, 8>(p, s);
    // (small ranges until there are two work-groups per CU: one row of 256000 words 7.1 us,
    // 9.1 with large ones; 200 rows of 32000 13.8, 18.1 with small ones)
    return p.M * p.V < (int64_t)kThreads * 8 * 512 ? launch_p<TYPE, true, 8>(p, s)
                                                   : launch_p<TYPE, true, 16>(p, s);
}

}  // namespace

hipError_t launch_adjust(const AdjustArgs& p, int32_t type, hipStream_t s)
{
    if (type == MQ_F32) return launch<MQ_F32>(p, s);
    return type == MQ_BF16 ? launch<MQ_BF16>(p, s) : launch<MQ_F16>(p, s);
}

}  // namespace mq
