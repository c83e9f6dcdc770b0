// The paged key/value cache and its batch of sequences on the device: where a
// token row or a tile of rows belongs, and where a position lies.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mq {

// Work-groups of a launch are fewer (of 256 threads, whose number is below 2^32).
constexpr int64_t kMaxBlocks = (int64_t)1 << 24;

struct KvArgs {
    int8_t* k;             // [pages][G][page][D]
    int8_t* v;             // [pages][G][D][page]
    int64_t pages;
    const int32_t* starts; // [B + 1]
    const int32_t* lens;   // [B]
    const int32_t* table;  // [B][ld]
    int64_t ld;
    int32_t B;
    int32_t G, D;
    int32_t shift;         // page = 1 << shift
};

// Entries of the page list that can name a page (an index past them has no
// place); a position is pos >> shift.
__device__ inline int64_t kv_page(const KvArgs& a, int32_t b, int64_t entry)
{
    if (entry < 0 || entry >= a.ld) return -1;
    const int64_t pg = a.table[(int64_t)b * a.ld + entry];
    return pg >= 0 && pg < a.pages ? pg : -1;
}

// The largest b in [0, B) with key(b) <= x (b = 0 if there is none), for an
// ascending key; the whole wave works on it, 64 probes a round, and every
// lane gets the answer.  Arrays that are not ascending give some b in range.
template <class Key>
__device__ inline int32_t find_seq(int32_t B, int64_t x, Key key)
{
    const int lane = threadIdx.x & 63;
    int32_t lo = 0, n = B;
    while (n > 1) {
        const int32_t step = (n + 63) >> 6;
        const int32_t off = lane * step;
        const uint64_t hit = __ballot(off < n && key(lo + off) <= x);
        const int32_t i = hit ? 63 - __builtin_clzll(hit) : 0;
        lo += i * step;
        n = min(step, n - i * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

hipError_t launch_rope_append(const KvArgs& kv, const int16_t* q, int64_t ldq, const int16_t* k,
                              int64_t ldk, const int8_t* v, int64_t ldv, int64_t T, int32_t H,
                              float aq, int32_t zq, float aqo, int32_t zqo, float ak, int32_t zk,
                              float ako, int32_t zko, const double* angles, int64_t positions,
                              int16_t* q_out, int64_t ldo, hipStream_t s);
hipError_t launch_paged_attn(const KvArgs& kv, const int16_t* q, int64_t ldq, int64_t T, int32_t H,
                             float q_scale, int32_t q_zp, float k_scale, float v_scale,
                             int32_t v_zp, float logit_scale, int64_t window, int64_t sinks,
                             float out_scale, int32_t out_zp, int32_t out_bits, void* y,
                             int64_t ldy, int64_t max_len, void* ws, int64_t ws_bytes,
                             hipStream_t s);
int64_t paged_attn_workspace(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D,
                             int64_t max_len);

}  // namespace mq
