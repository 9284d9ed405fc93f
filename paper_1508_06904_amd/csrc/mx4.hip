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

// ------------------------------------------------------------------ rows
// A workgroup has kRowTokens tokens of kRowBlocks blocks, four lanes for a block: a wave reads 512 adjacent channels of a
// token at a time. The scales turn round in LDS, so that those of adjacent tokens leave together.
constexpr int kRowTokens = 32, kRowBlocks = 16;

template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_mx4_rows_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t ts,
                                                                     uint8_t* __restrict__ codes, int64_t codes_stride,
                                                                     uint8_t* __restrict__ scales, int64_t scales_stride) {
    __shared__ uint8_t bytes[kRowBlocks][kRowTokens];
    const int64_t m0 = (int64_t)blockIdx.x * kRowTokens, b0 = (int64_t)blockIdx.y * kRowBlocks;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t b = b0 + (lane >> 2), k = b0 * kBlock + lane * 8;
    constexpr int PER = kRowTokens / (kThreads / 64);      // tokens of a wave
    Eight<T> v[PER];
#pragma unroll
    for (int n = 0; n < PER; ++n)
        if (m0 + wave * PER + n < M) v[n].load(x + (m0 + wave * PER + n) * ts + k, K - k);
#pragma unroll
    for (int n = 0; n < PER; ++n) {
        const uint32_t byte = v[n].scale_byte_of_four();
        const int64_t m = m0 + wave * PER + n;
        if (m < M && b * kBlock < K) *reinterpret_cast<uint32_t*>(codes + m * codes_stride + k / 2) = v[n].codes(byte);
        if ((lane & 3) == 0) bytes[lane >> 2][wave * PER + n] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int n = threadIdx.x; n < kRowBlocks * kRowTokens; n += kThreads) {
        const int64_t m = m0 + n % kRowTokens, at = b0 + n / kRowTokens;
        if (m < M && at * kBlock < K) scales[at * scales_stride + m] = bytes[n / kRowTokens][n % kRowTokens];
    }
}

// ------------------------------------------------------------------ maps
// 16 lanes have 16 bytes each of one channel, 256 adjacent bytes; a lane has the 32 channels of a block of its
// tokens, so that a block's codes leave it as 16 bytes and its tokens' scales as one word, and nothing passes between
// lanes. The last tile ends with the last token, and computes what the one before it has over again.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_mx4_map_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t ks,
                                                                    uint8_t* __restrict__ codes, int64_t codes_stride,
                                                                    uint8_t* __restrict__ scales, int64_t scales_stride) {
    using Block = MapBlock<T>;
    const int64_t m = min(xcd_order(blockIdx.x, gridDim.x) * Block::kTokens, M - Block::kTokens) + (threadIdx.x & 15) * Block::V;
    const int64_t b = (int64_t)blockIdx.y * (kThreads / 16) + (threadIdx.x >> 4);
    if (b * kBlock >= K) return;
    Block v;
    v.load(x + m + b * kBlock * ks, ks, (int)min((int64_t)kBlock, K - b * kBlock));
    uint32_t byte[Block::V];
    v.scale_bytes(byte);
#pragma unroll
    for (int j = 0; j < Block::V; ++j)
        *reinterpret_cast<i32x4*>(codes + (m + j) * codes_stride + b * 16) = v.codes(j, byte[j]);
    struct {
        uint8_t b[Block::V];
    } all;
#pragma unroll
    for (int j = 0; j < Block::V; ++j) all.b[j] = (uint8_t)byte[j];
    __builtin_memcpy(scales + b * scales_stride + m, &all, sizeof all);
}

// Narrower maps: a thread for each block of a token.
template <typename T>
__global__ __launch_bounds__(kThreads) void quantize_mx4_narrow_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t ks,
                                                                       uint8_t* __restrict__ codes, int64_t codes_stride,
                                                                       uint8_t* __restrict__ scales, int64_t scales_stride) {
    const int64_t id = (int64_t)blockIdx.x * kThreads + threadIdx.x, b = id / M, m = id - b * M, k0 = b * kBlock;
    if (k0 >= K) return;
    uint32_t byte;
    *reinterpret_cast<i32x4*>(codes + m * codes_stride + b * 16) = block_codes(x + m + k0 * ks, ks, (int)min((int64_t)kBlock, K - k0), byte);
    scales[b * scales_stride + m] = (uint8_t)byte;
}

// ------------------------------------------------------------------ values
__device__ __forceinline__ float value_of(uint32_t word, int k, float scale, bool nan) {
    using f32x2 = __attribute__((ext_vector_type(2))) float;
    f32x2 v;
    switch (k / 2) {
        case 0: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 0); break;
        case 1: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 1); break;
        case 2: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 2); break;
        default: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, 3); break;
    }
    return nan ? __uint_as_float(0x7fc00000u) : v[k & 1];
}

// Rows: four lanes for a block, eight adjacent values each.
template <typename T>
__global__ __launch_bounds__(kThreads) void dequantize_mx4_rows_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ts) {
    const int64_t m0 = (int64_t)blockIdx.x * kRowTokens + (threadIdx.x >> 6) * (kRowTokens / (kThreads / 64));
    const int lane = threadIdx.x & 63;
    const int64_t b = (int64_t)blockIdx.y * kRowBlocks + (lane >> 2), k = (int64_t)blockIdx.y * kRowBlocks * kBlock + lane * 8;
    if (b * kBlock >= K) return;
#pragma unroll
    for (int n = 0; n < kRowTokens / (kThreads / 64); ++n) {
        const int64_t m = m0 + n;
        if (m >= R.rows) return;
        const uint32_t word = *reinterpret_cast<const uint32_t*>(R.codes + m * R.stride + k / 2);
        const uint32_t byte = R.scales[b * R.scales_stride + m];
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = value_of(word, i, scale_operand(byte), byte == 255u);
        store_values(out + m * ts + k, v, k, K, 0);
    }
}

// Maps: a block of 4 or 8 adjacent tokens for a lane, and a wave's tokens are adjacent, so that it writes 1 KB of a channel
// at a time.  1.88 million tokens of 512 channels to binary32: 1242 us; 256 bytes at a time 1515, 4 KB (four waves side by
// side) 1380.
constexpr int kMapBlocks = 4, kMapTokens = 64;        // of a workgroup: blocks, lanes side by side

template <typename T>
__global__ __launch_bounds__(kMapBlocks * kMapTokens) void dequantize_mx4_map_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ks) {
    constexpr int V = 16 / (int)sizeof(T);
    const int64_t m = (xcd_order(blockIdx.x, gridDim.x) * kMapTokens + threadIdx.x % kMapTokens) * V;
    const int64_t b = (int64_t)blockIdx.y * kMapBlocks + threadIdx.x / kMapTokens;
    if (b * kBlock >= K || m >= R.rows) return;
    i32x4 w[V];
    uint32_t byte[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int64_t at = min(m + j, R.rows - 1);
        w[j] = *reinterpret_cast<const i32x4*>(R.codes + at * R.stride + b * 16);
        byte[j] = R.scales[b * R.scales_stride + at];
    }
    const int n = (int)min((int64_t)kBlock, K - b * kBlock);
    T* p = out + m + b * kBlock * ks;
#pragma unroll
    for (int k = 0; k < kBlock; ++k) {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = value_of((uint32_t)w[j][k / 8], k % 8, scale_operand(byte[j]), byte[j] == 255u);
        if (k < n) store_values(p + k * ks, v, m, R.rows, 0);
    }
}

// A launch has fewer than 2^32 threads, and 65535 workgroups along y, so large calls take several: `tokens` at a
// time, and so many blocks.
constexpr int64_t kGridY = 65535;
int64_t slab_tokens(int64_t B, int64_t blocks_y) {
    const int64_t y = std::min(ceil_div64(B, blocks_y), kGridY);
    return std::max<int64_t>(64, ((int64_t)1 << 23) / y) * 32;
}

template <typename T>
hipError_t run_quantize(const T* x, int64_t M, int64_t K, int64_t ts, int64_t ks, uint8_t* codes, int64_t cs, uint8_t* scales,
                        int64_t ss, hipStream_t s) {
    const bool map = ks != 1 && K > 1, narrow = map && M < MapBlock<T>::kTokens;
    const int64_t B = blocks_of(K);
    if (narrow) {
        const int64_t slab_b = (int64_t)1 << 24;        // (of fewer than 128 tokens)
        for (int64_t b = 0; b < B; b += slab_b) {
            const int64_t k = b * kBlock, channels = std::min(K - k, slab_b * kBlock);
            const dim3 grid((unsigned)ceil_div64(M * blocks_of(channels), kThreads));
            quantize_mx4_narrow_kernel<T><<<grid, kThreads, 0, s>>>(x + k * ks, M, channels, ks, codes + b * 16, cs, scales + b * ss, ss);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    const int64_t per_y = map ? kThreads / 16 : kRowBlocks, slab_b = kGridY * per_y, slab = slab_tokens(B, per_y);
    for (int64_t b = 0; b < B; b += slab_b) {
        const int64_t n_b = std::min(B - b, slab_b), k = b * kBlock;
        for (int64_t m = 0; m < M; m += slab) {
            int64_t n = std::min(M - m, slab), m0 = m;
            if (map && n < MapBlock<T>::kTokens) m0 = M - MapBlock<T>::kTokens, n = MapBlock<T>::kTokens;
            const T* p = x + m0 * (map ? 1 : ts) + k * (map ? ks : 1);
            uint8_t *c = codes + m0 * cs + b * 16, *sc = scales + b * ss + m0;
            const dim3 grid((unsigned)ceil_div64(n, map ? MapBlock<T>::kTokens : kRowTokens), (unsigned)ceil_div64(n_b, per_y));
            const int64_t channels = std::min(K - k, slab_b * kBlock);
            if (map) quantize_mx4_map_kernel<T><<<grid, kThreads, 0, s>>>(p, n, channels, ks, c, cs, sc, ss);
            else quantize_mx4_rows_kernel<T><<<grid, kThreads, 0, s>>>(p, n, channels, ts, c, cs, sc, ss);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_dequantize(const Mx4Rows& R, int64_t K, T* out, int64_t ts, int64_t ks, bool map, hipStream_t s) {
    constexpr int kTokens = kMapTokens * (16 / (int)sizeof(T));
    const int64_t B = blocks_of(K), per_y = map ? kMapBlocks : kRowBlocks, slab_b = kGridY * per_y;
    const int64_t slab = slab_tokens(B, per_y);  // (tiles of at least 256 tokens: fewer threads than rows have)
    for (int64_t b = 0; b < B; b += slab_b) {
        const int64_t n_b = std::min(B - b, slab_b), k = b * kBlock, channels = std::min(K - k, slab_b * kBlock);
        for (int64_t m = 0; m < R.rows; m += slab) {
            const Mx4Rows P = {R.codes + m * R.stride + b * 16, R.stride, R.scales + b * R.scales_stride + m, R.scales_stride,
                               std::min(R.rows - m, slab)};
            const dim3 grid((unsigned)ceil_div64(P.rows, map ? kTokens : kRowTokens), (unsigned)ceil_div64(n_b, per_y));
            T* p = out + m * (map ? 1 : ts) + k * (map ? ks : 1);
            if (map) dequantize_mx4_map_kernel<T><<<grid, kMapBlocks * kMapTokens, 0, s>>>(P, channels, p, ks);
            else dequantize_mx4_rows_kernel<T><<<grid, kThreads, 0, s>>>(P, channels, p, ts);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_quantize_mx4(dss_dtype dt, const void* x, int64_t M, int K, int64_t token_stride, int64_t channel_stride,
                               uint8_t* codes, int64_t codes_stride, uint8_t* scales, int64_t scales_stride, hipStream_t s) {
    return dt == DSS_BF16 ? run_quantize((const uint16_t*)x, M, K, token_stride, channel_stride, codes, codes_stride, scales,
                                         scales_stride, s)
                          : run_quantize((const float*)x, M, K, token_stride, channel_stride, codes, codes_stride, scales,
                                         scales_stride, s);
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
    const Mx4Rows R = {codes, codes_stride, scales, scales_stride, M};
    dss_status s = check_mx4_rows(R, blocks_of(K), "tokens");
    if (s != DSS_OK) return s;
    s = check_outputs(M, K, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK || M == 0) return s;
    const bool map = is_map(M, K, out_token_stride, out_channel_stride);
    hipError_t e = out_dtype == DSS_BF16
                       ? run_dequantize(R, K, (uint16_t*)out, out_token_stride, out_channel_stride, map, stream)
                       : run_dequantize(R, K, (float*)out, out_token_stride, out_channel_stride, map, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "dequantize launch");
} catch (...) {
    return DSS_E_NOMEM;
}
