// Tokens in 8 bits: scale[m] = max_k |x[m][k]| / 127, code[m][k] = clamp(rint(x[m][k] / scale[m]), -127, 127).
//
// Bound by memory: every value is read once and its code written once.  Two
// layouts: rows (a token's channels adjacent) and maps (a channel's tokens
// adjacent, as the dense evaluation writes them).
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

constexpr int kThreads = 256;
// The largest of v over a token's LPR lanes.
template <int LPR>
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
#pragma unroll
    for (int d = (LPR < 64 ? LPR : 64) / 2; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, d));
    if constexpr (LPR > 64) {
        __shared__ uint32_t part[LPR / 64];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < LPR / 64; ++w) v = max(v, part[w]);
    }
    return v;
}

// Rows: LPR lanes hold a token of at most LPR * CH chunks in registers.  Codes are
// written up to channel Kp >= K (zeros from K on).
template <typename T, int LPR, int CH>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(const T* __restrict__ x, int64_t M, int K,
                                                                 int64_t token_stride, int8_t* __restrict__ codes,
                                                                 int64_t codes_stride, int Kp,
                                                                 float* __restrict__ scales) {
    constexpr int E = Chunk<T>::E;
    const int64_t m = (int64_t)blockIdx.x * (kThreads / LPR) + threadIdx.x / LPR;
    if (m >= M) return;                  // (whole tokens: with LPR > 64 the workgroup has one)
    const int lane = threadIdx.x % LPR;
    const T* row = x + m * token_stride;
    Chunk<T> c[CH];
    uint32_t top = 0;
    load_row(c, row, lane, LPR, K);
#pragma unroll
    for (int i = 0; i < CH; ++i)
#pragma unroll
        for (int k = 0; k < E; ++k) top = max(top, abs_bits(to_f32(c[i].v[k])));
    const float scale = scale_of(row_max<LPR>(top));
    if (lane == 0) scales[m] = scale;
    const Coder coder(scale);
    int8_t* out = codes + m * codes_stride;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = (i * LPR + lane) * E;
        if (at < Kp) store_codes(out + at, c[i], coder, Kp - at);
    }
}

// Rows longer than the registers hold: read twice, the second time from cache.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_long_rows_kernel(const T* __restrict__ x, int K,
                                                                      int64_t token_stride,
                                                                      int8_t* __restrict__ codes, int64_t codes_stride,
                                                                      int Kp, float* __restrict__ scales) {
    constexpr int E = Chunk<T>::E;
    const int64_t m = blockIdx.x;
    const T* row = x + m * token_stride;
    uint32_t top = 0;
    for (int64_t at = threadIdx.x * E; at < K; at += kThreads * E) {
        const Chunk<T> c = load_chunk(row + at, (int)(K - at));
#pragma unroll
        for (int k = 0; k < E; ++k) top = max(top, abs_bits(to_f32(c.v[k])));
    }
    const float scale = scale_of(row_max<kThreads>(top));
    if (threadIdx.x == 0) scales[m] = scale;
    const Coder coder(scale);
    int8_t* out = codes + m * codes_stride;
    for (int64_t at = threadIdx.x * E; at < Kp; at += kThreads * E)
        store_codes(out + at, load_chunk(row + at, (int)(K - at)), coder, (int)(Kp - at));
}

// Maps: a workgroup takes 64 adjacent tokens; a wave reads them of one channel at
// a time.  The second reading, from cache, goes through LDS, which turns 64
// channels of the 64 tokens round so that a token's codes leave together.
constexpr int kMapTokens = 64;
constexpr int kMapPitch = kMapTokens + 4;    // bytes of a token's row in LDS

template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_map_kernel(const T* __restrict__ x, int64_t M, int K,
                                                                int64_t channel_stride, int8_t* __restrict__ codes,
                                                                int64_t codes_stride, int Kp,
                                                                float* __restrict__ scales) {
    __shared__ uint32_t tops[kThreads];
    __shared__ __align__(16) int8_t tile[kMapTokens * kMapPitch];
    const int t = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t m0 = (int64_t)blockIdx.x * kMapTokens;
    const bool in = m0 + t < M;
    const T* col = x + m0 + t;
    uint32_t top = 0;
    if (in)
        for (int k = w; k < K; k += kThreads / 64) top = max(top, abs_bits(to_f32(col[k * channel_stride])));
    tops[threadIdx.x] = top;
    __syncthreads();
    top = max(max(tops[t], tops[64 + t]), max(tops[128 + t], tops[192 + t]));
    const float scale = scale_of(top);
    const Coder coder(scale);
    if (in && w == 0) scales[m0 + t] = scale;
    for (int k0 = 0; k0 < Kp; k0 += 64) {
        __syncthreads();
        for (int k = w; k < 64; k += kThreads / 64)
            tile[t * kMapPitch + k] = in && k0 + k < K ? coder.one(to_f32(col[(k0 + k) * channel_stride])) : 0;
        __syncthreads();
        // 4 lanes of 16 bytes for each token
        const int tok = threadIdx.x >> 2, at = (threadIdx.x & 3) * 16;
        if (m0 + tok < M && k0 + at < Kp) {
            int8_t* p = codes + (m0 + tok) * codes_stride + k0 + at;
            const int8_t* q = tile + tok * kMapPitch + at;
            const int n = min(16, Kp - k0 - at);
            if (n == 16) {
                uint32_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint32_t*>(q + 4 * j);
                __builtin_memcpy(p, v, 16);
            } else {
                for (int j = 0; j < n; ++j) p[j] = q[j];
            }
        }
    }
}

template <typename T, int LPR, int CH>
void run_rows(const T* x, int64_t M, int K, int64_t ts, int8_t* codes, int64_t cs, int Kp, float* scales, hipStream_t s) {
    quantize_rows_kernel<T, LPR, CH><<<dim3((unsigned)ceil_div64(M, kThreads / LPR)), kThreads, 0, s>>>(x, M, K, ts, codes,
                                                                                                       cs, Kp, scales);
}

template <typename T>
void run_quantize(const T* x, int64_t M, int K, int64_t ts, int64_t ks, int8_t* codes, int64_t cs, int Kp, float* scales,
                  hipStream_t s) {
    constexpr int E = Chunk<T>::E;
    if (ks != 1 && K > 1) {
        quantize_map_kernel<T><<<dim3((unsigned)ceil_div64(M, kMapTokens)), kThreads, 0, s>>>(x, M, K, ks, codes, cs, Kp,
                                                                                             scales);
        return;
    }
    // as many lanes for a token as leave each of them a few chunks to have in flight
    if (Kp <= 16 * E) run_rows<T, 16, 1>(x, M, K, ts, codes, cs, Kp, scales, s);
    else if (Kp <= 64 * E) run_rows<T, 16, 4>(x, M, K, ts, codes, cs, Kp, scales, s);
    else if (Kp <= 256 * E) run_rows<T, 64, 4>(x, M, K, ts, codes, cs, Kp, scales, s);
    else if (Kp <= 1024 * E) run_rows<T, 256, 4>(x, M, K, ts, codes, cs, Kp, scales, s);
    else if (Kp <= 4096 * E) run_rows<T, 256, 16>(x, M, K, ts, codes, cs, Kp, scales, s);
    else quantize_long_rows_kernel<T><<<dim3((unsigned)M), kThreads, 0, s>>>(x, K, ts, codes, cs, Kp, scales);
}

}  // namespace

hipError_t launch_quantize_tokens(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride,
                                  int64_t channel_stride, int8_t* codes, int64_t codes_stride, int Kp, float* scales,
                                  hipStream_t s) {
    for (int64_t m = 0; m < M; m += kSlabTokens) {
        const int64_t n = std::min(M - m, kSlabTokens), at = m * token_stride;
        int8_t* c = codes + m * codes_stride;
        if (dt == DSS_BF16)
            run_quantize((const uint16_t*)x + at, n, K, token_stride, channel_stride, c, codes_stride, Kp, scales + m, s);
        else
            run_quantize((const float*)x + at, n, K, token_stride, channel_stride, c, codes_stride, Kp, scales + m, s);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

dss_status check_tokens(const void* x, dss_dtype dtype, int64_t M, int32_t K, int64_t token_stride,
                        int64_t channel_stride) {
    if (dtype != DSS_F32 && dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", dtype);
    if (M < 0 || M > kMaxTokens || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels", (long long)M, K);
    if (token_stride < 0 || channel_stride < 0) return fail(DSS_E_INVALID, "negative stride");
    if ((channel_stride != 1 && K > 1) && (token_stride != 1 && M > 1))
        return fail(DSS_E_UNSUPPORTED, "neither the tokens nor the channels are adjacent (strides %lld, %lld)",
                    (long long)token_stride, (long long)channel_stride);
    if (M > 0 && (!x || (uintptr_t)x % dtype_size(dtype) != 0))
        return fail(DSS_E_INVALID, "x is NULL or not aligned to its elements");
    return DSS_OK;
}

}  // namespace dss

extern "C" dss_status dss_quantize_tokens(const void* x, dss_dtype dtype, int64_t M, int32_t K, int64_t token_stride,
                                          int64_t channel_stride, int8_t* codes, int64_t codes_stride, float* scales,
                                          hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    if (codes_stride < K) return fail(DSS_E_INVALID, "codes_stride %lld is less than %d", (long long)codes_stride, K);
    if (M == 0) return DSS_OK;
    if (!codes || !scales || (uintptr_t)scales % 4 != 0)
        return fail(DSS_E_INVALID, "codes or scales is NULL or not aligned to its elements");
    hipError_t e = launch_quantize_tokens(dtype, x, M, K, token_stride, channel_stride, codes, codes_stride, K, scales,
                                          stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "quantize launch");
} catch (...) {
    return DSS_E_NOMEM;
}
