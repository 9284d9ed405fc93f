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

// The checks of a layer's outputs and of its workspace, and whether the output is a map (as rows where both would do).
dss_status check_outputs(int64_t M, int32_t N, const void* out, dss_dtype out_dtype, int64_t out_token_stride,
                         int64_t out_channel_stride);
dss_status check_room(int64_t need, const void* workspace, int64_t workspace_bytes);
bool is_map(int64_t M, int32_t N, int64_t out_token_stride, int64_t out_channel_stride);

// A fully connected layer on codes (codes and scales unused where the kernel codes the tokens itself).
struct Layer {
    const int8_t* codes;
    int64_t codes_stride;
    const float* scales;
    int64_t M;
    const int8_t* weight;
    int64_t weight_stride;
    const float* weight_scales;
    int N, K;
    const float* bias;
    int act;
    void* out;
    int64_t ldo;                         // the output's stride that is not 1
    int map;                             // out is [N][M], not [M][N]
    int past;                            // the outputs go around the caches
};

// Whether outputs go around the caches: large ones whose rows are whole lines.  200000 x
// 1024 in bfloat16 from 512 channels: 280 us around them and 340 through them; 512 x 198025 in
// binary32 from 256, where rows end inside lines: 925 and 387.
inline bool outputs_past(int64_t M, int64_t N, int64_t ldo, const void* out, dss_dtype dt) {
    const int64_t es = (int64_t)dtype_size(dt);
    return M * N * es > ((int64_t)1 << 26) && ldo * es % 128 == 0 && (uintptr_t)out % 128 == 0;
}

// Tokens that are not codes yet.
struct Values {
    const void* x;
    dss_dtype dtype;
    int64_t token_stride, channel_stride;
};

// The layer for few tokens (matmul_few.hip): whether it runs there, and whether the
// kernel codes M tokens of K channels itself, with no workspace.
bool few_tokens(int64_t M, int N, int K);
hipError_t launch_matmul_few(const Layer& L, dss_dtype out_dtype, hipStream_t s);
bool codes_itself(int64_t M, int K);
hipError_t launch_linear_few(const Layer& L, const Values& V, dss_dtype out_dtype, hipStream_t s);

// The layer on many tokens of a map of few channels with few outputs, coded and
// multiplied in one launch (linear_tile.hip), and whether it runs there.
bool linear_in_tiles(int64_t M, int N, int K, bool map);
hipError_t launch_linear_tiles(const Layer& L, const Values& V, dss_dtype out_dtype, hipStream_t s);

// Codes and scales of M > 0 tokens; codes[m][K .. Kp-1] are written as zeros.
hipError_t launch_quantize_tokens(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride,
                                  int64_t channel_stride, int8_t* codes, int64_t codes_stride, int Kp, float* scales,
                                  hipStream_t s);

}  // namespace dss
