// The paged key/value cache with a scale for each block of tokens and head.
#pragma once

#include "kvcache.h"

namespace mq {

struct BlockCache {
    KvArgs kv;       // k [pages][G][page][D]; v [pages][G][page / 16][D][16]
    float* k_scale;  // [pages][G][page / block]
    float* v_scale;
    int32_t bshift;  // block = 1 << bshift, 16 <= block <= page
};

// Scale of head g in the block of `slot` of page pg.
__device__ inline int64_t scale_at(const BlockCache& c, int64_t pg, int32_t g, int32_t slot)
{
    return ((pg * c.kv.G + g) << (c.kv.shift - c.bshift)) + (slot >> c.bshift);
}

hipError_t launch_append_blocks(const BlockCache& c, const void* q, int64_t ldq, const void* k,
                                int64_t ldk, const void* v, int64_t ldv, int32_t type, int64_t T,
                                int32_t H, const double* angles, int64_t positions, void* q_out,
                                int64_t ldo, hipStream_t s);

int64_t attn_blocks_workspace(int64_t T, int64_t B, int32_t H, int32_t G, int32_t D,
                              int64_t max_len);
hipError_t launch_attn_blocks(const BlockCache& c, const void* q, int64_t ldq, int32_t type,
                              int64_t T, int32_t H, float logit_scale, int64_t window,
                              int64_t sinks, void* y, int64_t ldy, int64_t max_len, void* ws,
                              int64_t ws_bytes, hipStream_t s);

}  // namespace mq
