// Launches of the token quantizer and of the product with token scales.
#pragma once

#include "mq_internal.h"
#include "tokens.h"

namespace mq {

hipError_t launch_quantize_tokens(const void* x, int32_t type, int64_t M, int64_t K, int64_t ldx,
                                  int8_t* x_q, float* scale, int32_t* rowsum, int32_t* clear,
                                  int64_t clear_n, hipStream_t s);
// p: a, w, w_scale, w_zp, a_rowsum, bias, sizes and workspace; path resolved.
hipError_t launch_qlinear_tokens(const QLinearArgs& p, const TokenArgs& t, int32_t path,
                                 hipStream_t s);
// One token's product from its floating activations x, quantized by every
// work-group for itself; whether it is the faster form (else: quantize first).
bool one_token_fused(const QLinearArgs& p, const void* x);
// Whether 2 to 16 tokens go through the many tokens' tiles where the caller leaves the
// path open.
bool few_tokens_in_tiles(const QLinearArgs& p, int32_t y_type);
hipError_t launch_linear_one_token(const QLinearArgs& p, const TokenArgs& t, const void* x,
                                   int32_t type, hipStream_t s);

}  // namespace mq
