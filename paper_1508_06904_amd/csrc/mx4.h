// Internal declarations of the tokens in microscaled 4-bit floating point: their coding (mx4.hip)
// and their products with weights of the same kind (matmul_mx4.hip, few_mx4.hip).
#pragma once

#include "tokens.h"

namespace dss {

constexpr int kBlock = 32;               // channels that share a scale: 16 bytes of codes

inline int64_t blocks_of(int64_t K) { return (K + kBlock - 1) / kBlock; }

// Rows in 4 bits: codes[r * stride + 16 b ..], scales[b * scales_stride + r].
struct Mx4Rows {
    const uint8_t* codes;
    int64_t stride;
    const uint8_t* scales;
    int64_t scales_stride;
    int64_t rows;
};

// A fully connected layer (the tokens unused where the kernel codes them itself).
struct Mx4Layer {
    Mx4Rows tokens, weight;
    int B;                               // blocks of a row
    const float* bias;
    int act;
    void* out;
    int64_t ldo;                         // the output's stride that is not 1
    int map;                             // out is [N][M], not [M][N]
    int past;                            // the outputs go around the caches
};

// The checks of rows of B blocks, codes and scales.
dss_status check_mx4_rows(const Mx4Rows& R, int64_t B, const char* what);

// Tokens that are not codes yet.
struct Mx4Values {
    const void* x;
    dss_dtype dtype;
    int64_t channels, token_stride, channel_stride;
};

// Codes and scales of M > 0 tokens.
hipError_t launch_quantize_mx4(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride, int64_t channel_stride,
                               uint8_t* codes, int64_t codes_stride, uint8_t* scales, int64_t scales_stride, hipStream_t s);

// The layer on the tokens of a map, coded and multiplied in one launch (linear_mx4.hip), and whether it runs there.
bool linear_mx4_at_once(int64_t M, int64_t N, int64_t K, bool map);
hipError_t launch_linear_mx4(const Mx4Layer& L, const Mx4Values& X, dss_dtype out_dtype, hipStream_t s);

// The layer where one side has at most kFewRows rows (few_mx4.hip); and on so few tokens that the kernel codes them itself,
// and whether it does.  From 17 rows on two operands of few rows would be needed, and tiles are faster: 32 x 4096 to 4096 outputs 9.9
// us for 10.9, 32 x 9216 to 8192 17 for 31 (but 17 x 9216 to 512 14.9 for 10.1).
constexpr int kFewRows = 16;
hipError_t launch_few_mx4(const Mx4Layer& L, dss_dtype out_dtype, hipStream_t s);
bool few_codes_itself(int64_t M, int64_t K);
hipError_t launch_linear_few_mx4(const Mx4Layer& L, const Mx4Values& X, dss_dtype out_dtype, hipStream_t s);

}  // namespace dss
