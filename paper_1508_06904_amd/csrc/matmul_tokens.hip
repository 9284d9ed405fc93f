// Products of 8-bit tokens with 8-bit weights:
//   y[m][n] = act(scale[m] * weight_scale[n] * sum_k code[m][k] * weight[n][k] + bias[n]).
//
// The sums are exact: v_mfma_i32_16x16x64_i8 over 32-bit integers, whose range K
// <= 131071 keeps (128 * 128 * 131071 < 2^31).  Integers add in any order to the same bits,
// so tiles, and the division of K, are free to follow the sizes.
//
// D[i][j] = sum_k P[i][k] Q[j][k] with the output's adjacent axis as j: for rows
// P are the tokens and Q the weights, for dense maps the other way round.  In the
// matrix instruction Q's rows are the result's rows, so that a lane holds four
// adjacent outputs.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"

namespace dss {

namespace {

using i32x4 = __attribute__((ext_vector_type(4))) int;

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
};

// A NaN stays one (fmaxf would make it 0).
__device__ __forceinline__ float activate_nan(int act, float v) {
    if (act == DSS_ACT_RELU) return v < 0.f ? 0.f : v;
    if (act == DSS_ACT_TANH) return tanhf(v);
    return v;
}

__device__ __forceinline__ float output_of(int sum, float wscale, float scale, float bias, int act) {
    return activate_nan(act, (float)sum * wscale * scale + bias);
}

// ------------------------------------------------------------------ any sizes and strides
// 64 x 64 outputs for four waves of 16 (i) x 64 (j); 64 of K at a time through LDS.
constexpr int kTile = 64;
constexpr int kPitch = 64 + 16;

template <typename Tout>
__global__ __launch_bounds__(256) void matmul_any_kernel(Layer L, int tiles_j) {
    __shared__ __align__(16) int8_t lp[kTile * kPitch], lq[kTile * kPitch];
    const int8_t* P = L.map ? L.weight : L.codes;
    const int8_t* Q = L.map ? L.codes : L.weight;
    const int64_t ps = L.map ? L.weight_stride : L.codes_stride, qs = L.map ? L.codes_stride : L.weight_stride;
    const int64_t I = L.map ? L.N : L.M, J = L.map ? L.M : L.N;
    const int64_t i0 = (int64_t)(blockIdx.x / tiles_j) * kTile, j0 = (int64_t)(blockIdx.x % tiles_j) * kTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    i32x4 acc[4] = {};
    for (int k0 = 0; k0 < L.K; k0 += 64) {
        __syncthreads();
        for (int e = threadIdx.x; e < kTile * 64; e += 256) {
            const int r = e >> 6, k = e & 63;
            const bool in = k0 + k < L.K;
            lp[r * kPitch + k] = in && i0 + r < I ? P[(i0 + r) * ps + k0 + k] : 0;
            lq[r * kPitch + k] = in && j0 + r < J ? Q[(j0 + r) * qs + k0 + k] : 0;
        }
        __syncthreads();
        const i32x4 p = *reinterpret_cast<const i32x4*>(lp + (wave * 16 + (lane & 15)) * kPitch + (lane >> 4) * 16);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const i32x4 q = *reinterpret_cast<const i32x4*>(lq + (t * 16 + (lane & 15)) * kPitch + (lane >> 4) * 16);
            acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q, p, acc[t], 0, 0, 0);
        }
    }
    const int64_t i = i0 + wave * 16 + (lane & 15);
    if (i >= I) return;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int64_t j = j0 + t * 16 + (lane >> 4) * 4 + r;
            if (j >= J) continue;
            const int64_t m = L.map ? j : i;
            const int n = (int)(L.map ? i : j);
            const float y = output_of(acc[t][r], L.weight_scales[n], L.scales[m], L.bias ? L.bias[n] : 0.f, L.act);
            store_elem(static_cast<Tout*>(L.out) + i * L.ldo + j, y);
        }
}

hipError_t launch_matmul(const Layer& L, dss_dtype out_dtype, hipStream_t s) {
    for (int64_t m = 0; m < L.M; m += kSlabTokens) {
        Layer S = L;
        S.M = std::min(L.M - m, kSlabTokens);
        S.codes += m * L.codes_stride;
        S.scales += m;
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        const int64_t ti = ceil_div64(S.map ? S.N : S.M, kTile), tj = ceil_div64(S.map ? S.M : S.N, kTile);
        const dim3 grid((unsigned)(ti * tj));
        if (out_dtype == DSS_BF16) matmul_any_kernel<uint16_t><<<grid, 256, 0, s>>>(S, (int)tj);
        else matmul_any_kernel<float><<<grid, 256, 0, s>>>(S, (int)tj);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxK = 131071;
constexpr int kMaxN = 1 << 20;

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

// The codes' row length in a workspace: whole 16-byte units.
int padded_k(int K) { return (K + 15) / 16 * 16; }

// Checks of what dss_matmul_tokens and dss_linear_tokens share.
dss_status check_layer(int64_t M, const int8_t* weight, int64_t weight_stride, const float* weight_scales, int32_t N,
                       int32_t K, const float* bias, dss_act act, const void* out, dss_dtype out_dtype,
                       int64_t out_token_stride, int64_t out_channel_stride) {
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (act != DSS_ACT_NONE && act != DSS_ACT_RELU && act != DSS_ACT_TANH)
        return fail(DSS_E_INVALID, "unknown activation %d", act);
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (K > kMaxK)
        return fail(DSS_E_UNSUPPORTED, "a sum of %d products of 8-bit codes may leave 32 bits (at most %d)", K, kMaxK);
    if (weight_stride < K) return fail(DSS_E_INVALID, "weight_stride %lld is less than %d", (long long)weight_stride, K);
    const bool rows = (out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1);
    const bool map = (out_token_stride == 1 || M <= 1) && (out_channel_stride >= M || N == 1);
    if (!rows && !map)
        return fail(out_channel_stride == 1 || out_token_stride == 1 ? DSS_E_INVALID : DSS_E_UNSUPPORTED,
                    "output strides %lld (tokens) and %lld (channels)", (long long)out_token_stride,
                    (long long)out_channel_stride);
    if (!weight || !weight_scales || (uintptr_t)weight_scales % 4 != 0 || (uintptr_t)bias % 4 != 0)
        return fail(DSS_E_INVALID, "weight or weight_scales is NULL, or the scales or the bias are not aligned");
    if (M > 0 && (!out || (uintptr_t)out % dtype_size(out_dtype) != 0))
        return fail(DSS_E_INVALID, "out is NULL or not aligned to its elements");
    return DSS_OK;
}

int64_t workspace_bytes_of(int64_t M, int32_t N, int32_t K, bool from_codes) {
    (void)N;
    return from_codes ? 0 : align256(M * 4) + align256(M * padded_k(K));
}

dss_status check_room(int64_t need, const void* workspace, int64_t workspace_bytes) {
    if (need == 0) return DSS_OK;
    if (!workspace || ((uintptr_t)workspace & 255u) != 0)
        return fail(DSS_E_INVALID, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(DSS_E_SHAPE, "workspace of %lld bytes is smaller than the %lld bytes needed",
                    (long long)workspace_bytes, (long long)need);
    return DSS_OK;
}

// The output's orientation: as rows where both would do.
bool is_map(int64_t M, int32_t N, int64_t out_token_stride, int64_t out_channel_stride) {
    return !((out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1));
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_tokens_workspace(int64_t M, int32_t N, int32_t K, int32_t from_codes,
                                           int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    *workspace_bytes = workspace_bytes_of(M, N, K, from_codes != 0);
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_matmul_tokens(const int8_t* codes, int64_t codes_stride, const float* scales, int64_t M,
                                        const int8_t* weight, int64_t weight_stride, const float* weight_scales,
                                        int32_t N, int32_t K, const float* bias, dss_act act, void* out,
                                        dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                        void* workspace, int64_t workspace_bytes, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_layer(M, weight, weight_stride, weight_scales, N, K, bias, act, out, out_dtype,
                               out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    if (codes_stride < K) return fail(DSS_E_INVALID, "codes_stride %lld is less than %d", (long long)codes_stride, K);
    if (M == 0) return DSS_OK;
    if (!codes || !scales || (uintptr_t)scales % 4 != 0)
        return fail(DSS_E_INVALID, "codes or scales is NULL or not aligned to its elements");
    s = check_room(workspace_bytes_of(M, N, K, true), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const Layer L = {codes, codes_stride, scales, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out,
                     map ? out_channel_stride : out_token_stride, map};
    hipError_t e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_linear_tokens(const void* x, dss_dtype dtype, int64_t M, int64_t token_stride,
                                        int64_t channel_stride, const int8_t* weight, int64_t weight_stride,
                                        const float* weight_scales, int32_t N, int32_t K, const float* bias,
                                        dss_act act, void* out, dss_dtype out_dtype, int64_t out_token_stride,
                                        int64_t out_channel_stride, void* workspace, int64_t workspace_bytes,
                                        hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    s = check_layer(M, weight, weight_stride, weight_scales, N, K, bias, act, out, out_dtype, out_token_stride,
                    out_channel_stride);
    if (s != DSS_OK) return s;
    if (M == 0) return DSS_OK;
    s = check_room(workspace_bytes_of(M, N, K, false), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    float* scales = static_cast<float*>(workspace);
    int8_t* codes = static_cast<int8_t*>(workspace) + align256(M * 4);
    const int Kp = padded_k(K);
    hipError_t e = launch_quantize_tokens(dtype, x, M, K, token_stride, channel_stride, codes, Kp, Kp, scales, stream);
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const Layer L = {codes, Kp, scales, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out,
                     map ? out_channel_stride : out_token_stride, map};
    e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}
