// Tokens in 8 bits: scale[m] = max_k |x[m][k]| / 127, code[m][k] = clamp(rint(x[m][k] / scale[m]), -127, 127).
//
// Bound by memory: every value is read once and its code written once.  Two
// layouts: rows (a token's channels adjacent) and maps (a channel's tokens
// adjacent, as the dense evaluation writes them).  Measured, bytes in and out: 1.88 million tokens of
// 512 channels in binary32 as a map 0.98 to 1.00 ms (4.8 to 4.9 TB/s), as rows 0.88 ms (5.5 TB/s),
// in bfloat16 0.64 (4.5) and 0.51 ms (5.6); 8191 rows of 4097 in bfloat16 21 us (4.8 TB/s); a
// large copy runs at 5.07 TB/s.
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
    for (int i = 0; i < CH; ++i) top = raise(top, c[i]);
    const float scale = scale_of(row_max<LPR>(top_bits<T>(top)));
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
    for (int64_t at = threadIdx.x * E; at < K; at += kThreads * E) top = raise(top, load_chunk(row + at, (int)(K - at)));
    const float scale = scale_of(row_max<kThreads>(top_bits<T>(top)));
    if (threadIdx.x == 0) scales[m] = scale;
    const Coder coder(scale);
    int8_t* out = codes + m * codes_stride;
    for (int64_t at = threadIdx.x * E; at < Kp; at += kThreads * E)
        store_codes(out + at, load_chunk(row + at, (int)(K - at)), coder, (int)(Kp - at));
}

// Maps of at least a tile's tokens: see MapTile.  The last tile ends with the last
// token and leaves out what the one before it has.  Of more channels than a workgroup
// holds the values are read twice, the second time mostly from cache.  Channels are
// counted in unsigned 32 bits: K is below 2^31, and no count passes it by more than a
// span of channels.
template <typename T>
__global__ __launch_bounds__(kMapWaves * 64) void quantize_map_kernel(const T* __restrict__ x, int64_t M, int K,
                                                                      int64_t channel_stride,
                                                                      int8_t* __restrict__ codes, int64_t codes_stride,
                                                                      int Kp, float* __restrict__ scales) {
    using Tile = MapTile<T>;
    __shared__ uint32_t tops[kMapWaves * 64];
    const int64_t tile0 = xcd_order(blockIdx.x, gridDim.x) * Tile::kTokens, m0 = min(tile0, M - Tile::kTokens);
    const int first = (int)(tile0 - m0);
    const uint32_t channels = K, channels_out = Kp;
    const uint32_t span = (blockDim.x >> 6) * 64;      // channels held at once
    const uint32_t own_k = (threadIdx.x >> 4) * 16;
    Tile tile;
    uint32_t top[4] = {};
    for (uint32_t k0 = 0; k0 < channels; k0 += span) {
        tile.load(x + m0, channel_stride, k0 + own_k, channels);
        tile.raise_into(top);
    }
    Tile::meet(top, tops, 0, blockDim.x >> 6);
    const int t = (threadIdx.x & 15) * Tile::V;
    const int rounds = (int)((channels + span - 1) / span);
    for (int round = rounds - 1; round >= 0; --round) {
        // (the last span is still there)
        const uint32_t k = round * span + own_k;
        if (round != rounds - 1) tile.load(x + m0, channel_stride, k, channels);
#pragma unroll
        for (int j = 0; j < Tile::V; ++j) {
            const Coder coder(scale_of(Tile::bits(top, j)));
            if (t + j < first) continue;
            if (round == 0 && threadIdx.x < 16) scales[m0 + t + j] = coder.scale;
            uint32_t w[4];
            tile.codes(j, coder, w);
            int8_t* p = codes + (m0 + t + j) * codes_stride + k;
            if (k + 16 <= channels_out) {
                __builtin_memcpy(p, w, 16);
            } else {
#pragma unroll
                for (int b = 0; b < 16; ++b)
                    if (k + b < channels_out) p[b] = (int8_t)(w[b / 4] >> (8 * (b % 4)));
            }
        }
    }
}

// Narrower maps: a workgroup for each token, value by value; the tokens' lines meet in cache.
// 16 to 63 binary32 tokens of 9216 channels take 22 us: a chain of 36 loads, twice.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_narrow_map_kernel(const T* __restrict__ x, int K,
                                                                       int64_t channel_stride,
                                                                       int8_t* __restrict__ codes, int64_t codes_stride,
                                                                       int Kp, float* __restrict__ scales) {
    const int64_t m = blockIdx.x;
    uint32_t top = 0;
    for (int64_t k = threadIdx.x; k < K; k += kThreads) top = max(top, abs_bits(to_f32(x[m + k * channel_stride])));
    const Coder coder(scale_of(row_max<kThreads>(top)));
    if (threadIdx.x == 0) scales[m] = coder.scale;
    for (int64_t k = threadIdx.x; k < Kp; k += kThreads)
        codes[m * codes_stride + k] = k < K ? coder.one(to_f32(x[m + k * channel_stride])) : 0;
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
        if (M < MapTile<T>::kTokens) {
            quantize_narrow_map_kernel<T><<<dim3((unsigned)M), kThreads, 0, s>>>(x, K, ks, codes, cs, Kp, scales);
            return;
        }
        const int waves = (int)std::min<int64_t>(((int64_t)K + 63) / 64, kMapWaves);
        quantize_map_kernel<T><<<dim3((unsigned)ceil_div64(M, MapTile<T>::kTokens)), waves * 64, 0, s>>>(x, M, K, ks, codes,
                                                                                                      cs, Kp, scales);
        return;
    }
    // as many lanes for a token as leave each of them a few chunks to have in flight
    if (Kp <= 4 * E) run_rows<T, 4, 1>(x, M, K, ts, codes, cs, Kp, scales, s);
    else if (Kp <= 16 * E) run_rows<T, 16, 1>(x, M, K, ts, codes, cs, Kp, scales, s);
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
