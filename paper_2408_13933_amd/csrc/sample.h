// Drawing tokens from logits (sample.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mq {

// Workspace of launch_sample: for all rows (within its bound), or the least.
int64_t sample_workspace(int64_t M, int64_t V, bool least);
hipError_t launch_sample(const void* x, int32_t bits, int64_t M, int64_t V, int64_t ld, float alpha,
                         const float* temperature, const int32_t* top_k, const float* top_p,
                         const float* min_p, const float* u, int32_t* tokens, void* ws,
                         int64_t ws_bytes, hipStream_t s);

}  // namespace mq
