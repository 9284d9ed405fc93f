// Tokens in microscaled 4-bit floating point: in each block of 32 channels a scale
// X = 2^(floor(log2(max |x|)) - 2) and codes of the values +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} nearest to x / X.
//
// Bound by memory: every value is read once, its half byte and a 32nd of a scale's byte written once.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

constexpr int kThreads = 256;

// A thread for each block of a token, any strides; blocks of adjacent tokens are adjacent threads'.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_mx4_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t ts,
                                                                int64_t ks, uint8_t* __restrict__ codes,
                                                                int64_t codes_stride, uint8_t* __restrict__ scales,
                                                                int64_t scales_stride) {
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = id / M, m = id - b * M, k0 = b * kBlock;
    if (k0 >= K) return;
    const T* p = x + m * ts + k0 * ks;
    const int n = (int)min((int64_t)kBlock, K - k0);
    float v[kBlock];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kBlock; ++k) {
        v[k] = k < n ? to_f32(p[k * ks]) : 0.f;
        top = max(top, abs_bits(v[k]));
    }
    const uint32_t byte = scale_byte(top);
    i32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float e[8] = {v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3], v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]};
        w[j] = byte == 255u ? 0 : (int)eight_codes(e, scale_operand(byte));
    }
    *reinterpret_cast<i32x4*>(codes + m * codes_stride + b * 16) = w;
    scales[b * scales_stride + m] = (uint8_t)byte;
}

// The values of a block, any strides.
template <typename T>
__global__ __launch_bounds__(kThreads) void dequantize_mx4_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ts,
                                                                  int64_t ks) {
    using f32x2 = __attribute__((ext_vector_type(2))) float;
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = id / R.rows, m = id - b * R.rows, k0 = b * kBlock;
    if (k0 >= K) return;
    const i32x4 w = *reinterpret_cast<const i32x4*>(R.codes + m * R.stride + b * 16);
    const uint32_t byte = R.scales[b * R.scales_stride + m];
    const float scale = scale_operand(byte);
    const int n = (int)min((int64_t)kBlock, K - k0);
    T* p = out + m * ts + k0 * ks;
    auto put = [&](int k, f32x2 v) {
        if (byte == 255u) v[0] = v[1] = __uint_as_float(0x7fc00000u);
        if (k < n) store_elem(p + k * ks, v[0]);
        if (k + 1 < n) store_elem(p + (k + 1) * ks, v[1]);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        put(8 * j, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)w[j], scale, 0));
        put(8 * j + 2, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)w[j], scale, 1));
        put(8 * j + 4, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)w[j], scale, 2));
        put(8 * j + 6, __builtin_amdgcn_cvt_scalef32_pk_f32_fp4((uint32_t)w[j], scale, 3));
    }
}

// Tokens of a launch: fewer than 2^32 threads.
int64_t slab_tokens(int64_t B) { return ((int64_t)1 << 31) / B; }    // (B <= 2^26)

}  // namespace

hipError_t launch_quantize_mx4(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride, int64_t channel_stride,
                               uint8_t* codes, int64_t codes_stride, uint8_t* scales, int64_t scales_stride, hipStream_t s) {
    const int64_t B = blocks_of(K), slab = slab_tokens(B);
    for (int64_t m = 0; m < M; m += slab) {
        const int64_t n = std::min(M - m, slab), at = m * token_stride;
        const dim3 grid((unsigned)ceil_div64(n * B, kThreads));
        uint8_t* c = codes + m * codes_stride;
        if (dt == DSS_BF16)
            quantize_mx4_kernel<uint16_t><<<grid, kThreads, 0, s>>>((const uint16_t*)x + at, n, K, token_stride, channel_stride, c,
                                                                    codes_stride, scales + m, scales_stride);
        else
            quantize_mx4_kernel<float><<<grid, kThreads, 0, s>>>((const float*)x + at, n, K, token_stride, channel_stride, c,
                                                                 codes_stride, scales + m, scales_stride);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

dss_status check_mx4_rows(const Mx4Rows& R, int64_t B, const char* what) {
    if (R.stride < 16 * B || (R.stride % 16 != 0 && R.rows > 1))
        return fail(DSS_E_INVALID, "%s: a row stride of %lld bytes for %lld blocks of 16", what, (long long)R.stride, (long long)B);
    if (R.scales_stride < R.rows && B > 1)
        return fail(DSS_E_INVALID, "%s: a scale stride of %lld for %lld rows", what, (long long)R.scales_stride, (long long)R.rows);
    if (R.rows > 0 && (!R.codes || !R.scales || (uintptr_t)R.codes % 16 != 0))
        return fail(DSS_E_INVALID, "%s: codes or scales are NULL, or the codes not at a unit of 16 bytes", what);
    return DSS_OK;
}

}  // namespace dss

extern "C" dss_status dss_quantize_blocks(const void* x, dss_dtype dtype, int64_t M, int32_t K, int64_t token_stride,
                                       int64_t channel_stride, uint8_t* codes, int64_t codes_stride, uint8_t* scales,
                                       int64_t scales_stride, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    s = check_mx4_rows({codes, codes_stride, scales, scales_stride, M}, blocks_of(K), "tokens");
    if (s != DSS_OK || M == 0) return s;
    hipError_t e = launch_quantize_mx4(dtype, x, M, K, token_stride, channel_stride, codes, codes_stride, scales, scales_stride,
                                       stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "quantize launch");
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_dequantize_blocks(const uint8_t* codes, int64_t codes_stride, const uint8_t* scales,
                                         int64_t scales_stride, int64_t M, int32_t K, void* out, dss_dtype out_dtype,
                                         int64_t out_token_stride, int64_t out_channel_stride, hipStream_t stream) try {
    using namespace dss;
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (M < 0 || M > kMaxTokens || K < 1) return fail(DSS_E_INVALID, "%lld tokens of %d channels", (long long)M, K);
    const int64_t B = blocks_of(K), slab = slab_tokens(B);
    dss_status s = check_mx4_rows({codes, codes_stride, scales, scales_stride, M}, B, "tokens");
    if (s != DSS_OK) return s;
    s = check_outputs(M, K, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    for (int64_t m = 0; m < M; m += slab) {
        const Mx4Rows R = {codes + m * codes_stride, codes_stride, scales + m, scales_stride, std::min(M - m, slab)};
        const dim3 grid((unsigned)ceil_div64(R.rows * B, kThreads));
        if (out_dtype == DSS_BF16)
            dequantize_mx4_kernel<uint16_t><<<grid, kThreads, 0, stream>>>(R, K, (uint16_t*)out + m * out_token_stride, out_token_stride,
                                                                           out_channel_stride);
        else
            dequantize_mx4_kernel<float><<<grid, kThreads, 0, stream>>>(R, K, (float*)out + m * out_token_stride, out_token_stride,
                                                                        out_channel_stride);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "dequantize launch");
    }
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}
