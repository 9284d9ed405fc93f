// Fully connected layers in microscaled 4-bit floating point:
//   y[m][n] = act(sum_b X[b][m] W[b][n] sum_{k in b} q[m][k] v[n][k] + bias[n]),
// on v_mfma_scale_f32_16x16x128_f8f6f4, whose binary32 sums take the blocks' scales with them.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

// The layer on codes.
hipError_t launch_matmul(const Mx4Layer& L, dss_dtype out_dtype, hipStream_t s) {
    if (L.tokens.rows <= kFewRows || L.weight.rows <= kFewRows) return launch_few_mx4(L, out_dtype, s);
    for (int64_t m = 0; m < L.tokens.rows; m += kFewRows) {
        Mx4Layer S = L;
        S.tokens.rows = std::min<int64_t>(kFewRows, L.tokens.rows - m);
        S.tokens.codes += m * L.tokens.stride;
        S.tokens.scales += m;
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        const hipError_t e = launch_few_mx4(S, out_dtype, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxN = 1 << 20;
constexpr int kMaxBlocks = 1 << 26;

// Checks of what dss_matmul_blocks and dss_linear_blocks share.
dss_status check_layer(int64_t M, const Mx4Rows& W, int64_t B, const float* bias, dss_act act, const void* out,
                       dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride) {
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (act != DSS_ACT_NONE && act != DSS_ACT_RELU && act != DSS_ACT_TANH)
        return fail(DSS_E_INVALID, "unknown activation %d", act);
    if (M < 0 || M > kMaxTokens || W.rows < 1 || W.rows > kMaxN || B < 1 || B > kMaxBlocks)
        return fail(DSS_E_INVALID, "%lld tokens of %lld blocks, %lld outputs", (long long)M, (long long)B, (long long)W.rows);
    dss_status s = check_mx4_rows(W, B, "weight");
    if (s != DSS_OK) return s;
    if ((uintptr_t)bias % 4 != 0) return fail(DSS_E_INVALID, "bias is not aligned to its elements");
    return check_outputs(M, (int32_t)W.rows, out, out_dtype, out_token_stride, out_channel_stride);
}

// The tokens' codes and scales.
int64_t workspace_bytes_of(int64_t M, int64_t B) { return align256(M * B * 16) + align256(M * B); }

Mx4Layer layer_of(const Mx4Rows& tokens, const Mx4Rows& weight, int64_t B, const float* bias, dss_act act, void* out,
                  dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride) {
    const bool map = is_map(tokens.rows, (int32_t)weight.rows, out_token_stride, out_channel_stride);
    const int64_t ldo = map ? out_channel_stride : out_token_stride;
    return {tokens, weight, (int)B, bias, (int)act, out, ldo, map, outputs_past(tokens.rows, weight.rows, ldo, out, out_dtype)};
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_blocks_workspace(int64_t M, int32_t N, int32_t K, dss_token_source source,
                                        int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (source != DSS_TOKENS_ROWS && source != DSS_TOKENS_MAP && source != DSS_TOKENS_CODES)
        return fail(DSS_E_INVALID, "unknown token source %d", (int)source);
    if (source != DSS_TOKENS_CODES && M > ((int64_t)1 << 62) / (blocks_of(K) * 17))
        return fail(DSS_E_INVALID, "the codes of %lld tokens of %d channels", (long long)M, K);
    *workspace_bytes = source == DSS_TOKENS_CODES ? 0 : workspace_bytes_of(M, blocks_of(K));
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_matmul_blocks(const uint8_t* codes, int64_t codes_stride, const uint8_t* scales, int64_t scales_stride,
                                     int64_t M, const uint8_t* weight, int64_t weight_stride, const uint8_t* weight_scales,
                                     int64_t weight_scales_stride, int32_t N, int32_t blocks, const float* bias, dss_act act,
                                     void* out, dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                     hipStream_t stream) try {
    using namespace dss;
    const Mx4Rows T = {codes, codes_stride, scales, scales_stride, M};
    const Mx4Rows W = {weight, weight_stride, weight_scales, weight_scales_stride, N};
    dss_status s = check_layer(M, W, blocks, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    s = check_mx4_rows(T, blocks, "tokens");
    if (s != DSS_OK || M == 0) return s;
    const Mx4Layer L = layer_of(T, W, blocks, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    hipError_t e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_linear_blocks(const void* x, dss_dtype dtype, int64_t M, int64_t token_stride, int64_t channel_stride,
                                     const uint8_t* weight, int64_t weight_stride, const uint8_t* weight_scales,
                                     int64_t weight_scales_stride, int32_t N, int32_t K, const float* bias, dss_act act,
                                     void* out, dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                     void* workspace, int64_t workspace_bytes, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    const int64_t B = blocks_of(K);
    const Mx4Rows W = {weight, weight_stride, weight_scales, weight_scales_stride, N};
    s = check_layer(M, W, B, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK || M == 0) return s;
    int64_t need = 0;
    s = dss_blocks_workspace(M, N, K, channel_stride != 1 && K > 1 ? DSS_TOKENS_MAP : DSS_TOKENS_ROWS, &need);
    if (s != DSS_OK) return s;
    s = check_room(need, workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + align256(M * B * 16);
    hipError_t e = launch_quantize_mx4(dtype, x, M, K, token_stride, channel_stride, codes, B * 16, scales, M, stream);
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    const Mx4Layer L = layer_of({codes, B * 16, scales, M, M}, W, B, bias, act, out, out_dtype, out_token_stride,
                                out_channel_stride);
    e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}
