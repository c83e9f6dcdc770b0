// Launch of the adjustments of logits before a draw.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace mq {

struct AdjustArgs {
    void* x;
    int64_t M, V, ld;
    const int32_t* history;  // [M][ldh], or nullptr
    int64_t ldh, cols;
    const int32_t* hist_lens;
    const int32_t* prompt_lens;  // or nullptr: 0
    const float* repetition;     // each or nullptr: 1, 0, 0
    const float* presence;
    const float* frequency;
    const int32_t* bias_starts;  // [M + 1], or nullptr
    const int32_t* bias_tokens;
    const float* bias_values;
    int64_t bias_n;
    const uint32_t* mask;  // [M][ldm], or nullptr
    int64_t ldm;
};

// hipErrorInvalidConfiguration: more work-groups than a launch may have
hipError_t launch_adjust(const AdjustArgs& p, int32_t type, hipStream_t s);

}  // namespace mq
