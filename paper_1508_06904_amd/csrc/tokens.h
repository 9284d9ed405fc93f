// Internal declarations of the 8-bit tokens: their coding (tokens.hip) and their
// products with 8-bit weights (matmul_tokens.hip).
#pragma once

#include "dss_internal.h"

namespace dss {

constexpr int64_t kMaxTokens = (int64_t)1 << 40;
// Tokens of one launch: up to 1024 threads for each, and a launch has fewer than 2^32.
constexpr int64_t kSlabTokens = (int64_t)1 << 21;

// The checks of x that dss_quantize_tokens and dss_linear_tokens share.
dss_status check_tokens(const void* x, dss_dtype dtype, int64_t M, int32_t K, int64_t token_stride,
                        int64_t channel_stride);

// Codes and scales of M > 0 tokens; codes[m][K .. Kp-1] are written as zeros.
hipError_t launch_quantize_tokens(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride,
                                  int64_t channel_stride, int8_t* codes, int64_t codes_stride, int Kp, float* scales,
                                  hipStream_t s);

}  // namespace dss
