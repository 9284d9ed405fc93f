// Tokens in microscaled 4-bit floating point: in each block of 32 channels a scale
// X = 2^(floor(log2(max |x|)) - 2) and codes of the values +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} nearest to x / X.
//
// Bound by memory: every value is read once, its half byte and a 32nd of a scale's byte written once.  1.88 million tokens of 512
// binary32 channels of a map: 876 us, 5.0 TB/s, as fast as a large copy; 8191 rows of 4097 bfloat16 channels: 18 us.
#include <algorithm>
#include <type_traits>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

constexpr int kThreads = 256;

// ------------------------------------------------------------------ rows
// A workgroup has BLOCKS blocks of its tokens, four lanes for a block: a wave reads 512 adjacent channels of a
// token at a time, or 128 of four tokens that have no more. The scales turn round in LDS, so that those of adjacent tokens
// leave together.
constexpr int kRowBlocks = 512;          // of a workgroup, of all its tokens
constexpr int kFewBlocks = 4;            // of a token, at most, where a workgroup has four times the tokens

template <typename T, int BLOCKS>
__global__ __launch_bounds__(kThreads) void quantize_mx4_rows_kernel(const T* __restrict__ x, int64_t M, int64_t K, int64_t ts,
                                                                     uint8_t* __restrict__ codes, int64_t codes_stride,
                                                                     uint8_t* __restrict__ scales, int64_t scales_stride) {
    constexpr int TOKENS = kRowBlocks / BLOCKS, PER = kRowBlocks * 4 / kThreads;
    __shared__ uint8_t bytes[BLOCKS][TOKENS];
    const int64_t m0 = (int64_t)blockIdx.x * TOKENS, b0 = (int64_t)blockIdx.y * BLOCKS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quarter = lane % (BLOCKS * 4), block = quarter >> 2;
    const int64_t b = b0 + block, k = b0 * kBlock + quarter * 8;
    constexpr int AT_ONCE = 16 / BLOCKS;                   // tokens of a wave's load
    const int own = wave * PER * AT_ONCE + (AT_ONCE > 1 ? lane / (BLOCKS * 4) : 0);
    const int64_t m_own = m0 + own;
    Eight<T> v[PER];
#pragma unroll
    for (int n = 0; n < PER; ++n)
        if (m_own + n * AT_ONCE < M) v[n].load(x + (m_own + n * AT_ONCE) * ts + k, K - k);
#pragma unroll
    for (int n = 0; n < PER; ++n) {
        const uint32_t byte = v[n].scale_byte_of_four();
        const int64_t m = m_own + n * AT_ONCE;
        if (m < M && b * kBlock < K) *reinterpret_cast<uint32_t*>(codes + m * codes_stride + k / 2) = v[n].codes(byte);
        if ((quarter & 3) == 0) bytes[block][own + n * AT_ONCE] = (uint8_t)byte;
    }
    __syncthreads();
#pragma unroll
    for (int n = threadIdx.x; n < kRowBlocks; n += kThreads) {
        const int64_t m = m0 + n % TOKENS, at = b0 + n / TOKENS;
        if (m < M && at * kBlock < K) scales[at * scales_stride + m] = bytes[n / TOKENS][n % TOKENS];
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
    *reinterpret_cast<i32x4*>(codes + m * codes_stride + b * 16) =
        block_codes(x + m + k0 * ks, ks, (int)min((int64_t)kBlock, K - k0), byte);
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

// Rows: 16 bytes of values for a lane, so that a wave writes 1 KB at a time, around the caches where rows are whole lines.
// The scales of a workgroup's tokens and blocks come through LDS: of a block they are adjacent, of a token they are not.
// 1.88 million tokens of 512 channels to binary32: 743 us; with 32 bytes for a lane, which are two stores of half the lines, and scales
// from memory 1815.  (A fill of the values takes 560.)
template <typename T, int BLOCKS>
__global__ __launch_bounds__(kThreads) void dequantize_mx4_rows_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ts, int past) {
    constexpr int V = 16 / (int)sizeof(T), TOKENS = kRowBlocks / BLOCKS, PER = kRowBlocks * (kBlock / V) / kThreads;
    using Word = std::conditional_t<V == 4, uint16_t, uint32_t>;         // V codes
    __shared__ uint8_t bytes[BLOCKS][TOKENS];
    const int64_t m0 = (int64_t)blockIdx.x * TOKENS, b0 = (int64_t)blockIdx.y * BLOCKS;
#pragma unroll
    for (int n = threadIdx.x; n < kRowBlocks; n += kThreads) {
        const int64_t m = m0 + n % TOKENS, at = b0 + n / TOKENS;
        bytes[n / TOKENS][n % TOKENS] = m < R.rows && at * kBlock < K ? R.scales[at * R.scales_stride + m] : (uint8_t)0;
    }
    // A lane's pieces of V values: TURNS of a token that has ROW, or one of each AT_ONCE tokens.
    constexpr int ROW = BLOCKS * kBlock / V, TURNS = ROW > 64 ? ROW / 64 : 1, AT_ONCE = ROW > 64 ? 1 : 64 / ROW, N = PER / TURNS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int own = wave * N * AT_ONCE + (AT_ONCE > 1 ? lane / ROW : 0), place = AT_ONCE > 1 ? lane % ROW : lane;
    Word w[N][TURNS];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t m = m0 + own + n * AT_ONCE, k = b0 * kBlock + (t * 64 + place) * V;
            w[n][t] = m < R.rows && k < K ? *reinterpret_cast<const Word*>(R.codes + m * R.stride + k / 2) : (Word)0;
        }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int64_t m = m0 + own + n * AT_ONCE, k = b0 * kBlock + (t * 64 + place) * V;
            if (m >= R.rows || k >= K) continue;
            const uint32_t byte = bytes[(t * 64 + place) * V / kBlock][own + n * AT_ONCE];
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = value_of(w[n][t], i, scale_operand(byte), byte == 255u);
            store_values(out + m * ts + k, v, k, K, past);
        }
}

// Maps whose rows are whole lines of 128 bytes: a block of 4 or 8 adjacent tokens for a lane, and a wave's tokens are adjacent, so
// that it writes 1 KB of a channel at a time, around the caches.
constexpr int kMapWaves = 4;             // of a workgroup, adjacent blocks of the same tokens

template <typename T>
__global__ __launch_bounds__(kMapWaves * 64) void dequantize_mx4_whole_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ks) {
    constexpr int V = 16 / (int)sizeof(T);
    const int64_t m = (xcd_order(blockIdx.x, gridDim.x) * 64 + (threadIdx.x & 63)) * V;
    const int64_t b = (int64_t)blockIdx.y * kMapWaves + (threadIdx.x >> 6);
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
        if (k < n) store_values(p + k * ks, v, m, R.rows, 1);
    }
}

// Other maps: a channel's lines start at any token. A wave writes whole ones all the same, 256 tokens of a channel at a time: it
// has a line's tokens more, a block of each in LDS, from where a lane takes those of the channel's lines.  With its tokens in registers
// and the lines as they come 1.88 million tokens of 512 channels took 1194 us for 870 (bfloat16 642 for 591); where
// rows are whole lines the detour through LDS costs (884 for 870, but 518 for 599 of bfloat16, and 10.4 for 14.0 of 20000 tokens).
template <typename T>
struct MapLines {
    // (8 of bfloat16 for a lane would read 32 bytes of LDS 32 bytes apart, twice over the same banks: 829 us for 518)
    static constexpr int V = 4, kTokens = 64 * V, kLine = 128 / (int)sizeof(T), kAll = kTokens + kLine;
    uint32_t words[4][kAll];             // of eight codes each
    uint32_t scales[kAll];
};

template <typename T>
__global__ __launch_bounds__(kMapWaves * 64) void dequantize_mx4_map_kernel(Mx4Rows R, int64_t K, T* __restrict__ out, int64_t ks) {
    using Lines = MapLines<T>;
    constexpr int V = Lines::V;
    __shared__ Lines lines[kMapWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int64_t m0 = xcd_order(blockIdx.x, gridDim.x) * Lines::kTokens, b = (int64_t)blockIdx.y * kMapWaves + wave;
    const bool there = b * kBlock < K;
    Lines& own = lines[wave];
    if (there) {
#pragma unroll
        for (int t = lane; t < Lines::kAll; t += 64) {
            const int64_t m = min(m0 + t, R.rows - 1);
            const i32x4 w = *reinterpret_cast<const i32x4*>(R.codes + m * R.stride + b * 16);
#pragma unroll
            for (int i = 0; i < 4; ++i) own.words[i][t] = (uint32_t)w[i];
            own.scales[t] = (uint32_t)R.scales[b * R.scales_stride + m] << 23;
        }
    }
    __syncthreads();
    if (!there) return;
    const int n = (int)min((int64_t)kBlock, K - b * kBlock);
    T* p = out + m0 + b * kBlock * ks;
#pragma unroll 8
    for (int k = 0; k < kBlock; ++k, p += ks) {
        if (k >= n) break;
        const int shift = (int)(-(uintptr_t)p % 128 / sizeof(T)), at = shift + lane * V;
        auto value = [&](uint32_t word, uint32_t scale) { return value_of(word, k % 8, __uint_as_float(scale), scale == 255u << 23); };
        uint32_t w[V], x[V];
        __builtin_memcpy(w, &own.words[k / 8][at], sizeof w);
        __builtin_memcpy(x, &own.scales[at], sizeof x);
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = value(w[j], x[j]);
        store_values(p + at, v, m0 + at, R.rows, 1);
        // the first tokens' part of a line
        if (m0 == 0 && lane < min((int64_t)shift, R.rows)) store_elem(p + lane, value(own.words[k / 8][lane], own.scales[lane]));
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
    const int64_t row_blocks = B <= kFewBlocks ? kFewBlocks : 16, per_y = map ? kThreads / 16 : row_blocks;
    const int64_t slab_b = kGridY * per_y, slab = slab_tokens(B, per_y), tokens = map ? MapBlock<T>::kTokens : kRowBlocks / row_blocks;
    for (int64_t b = 0; b < B; b += slab_b) {
        const int64_t n_b = std::min(B - b, slab_b), k = b * kBlock;
        for (int64_t m = 0; m < M; m += slab) {
            int64_t n = std::min(M - m, slab), m0 = m;
            if (map && n < MapBlock<T>::kTokens) m0 = M - MapBlock<T>::kTokens, n = MapBlock<T>::kTokens;
            const T* p = x + m0 * (map ? 1 : ts) + k * (map ? ks : 1);
            uint8_t *c = codes + m0 * cs + b * 16, *sc = scales + b * ss + m0;
            const dim3 grid((unsigned)ceil_div64(n, tokens), (unsigned)ceil_div64(n_b, per_y));
            const int64_t channels = std::min(K - k, slab_b * kBlock);
            if (map) quantize_mx4_map_kernel<T><<<grid, kThreads, 0, s>>>(p, n, channels, ks, c, cs, sc, ss);
            else if (row_blocks == 16) quantize_mx4_rows_kernel<T, 16><<<grid, kThreads, 0, s>>>(p, n, channels, ts, c, cs, sc, ss);
            else quantize_mx4_rows_kernel<T, kFewBlocks><<<grid, kThreads, 0, s>>>(p, n, channels, ts, c, cs, sc, ss);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
    }
    return hipSuccess;
}

template <typename T>
hipError_t run_dequantize(const Mx4Rows& R, int64_t K, T* out, int64_t ts, int64_t ks, bool map, hipStream_t s) {
    const int64_t B = blocks_of(K), row_blocks = B <= kFewBlocks ? kFewBlocks : 16, per_y = map ? kMapWaves : row_blocks;
    const int64_t slab_b = kGridY * per_y;
    const bool whole = (map ? ks : ts) * (int64_t)sizeof(T) % 128 == 0 && (uintptr_t)out % 128 == 0;
    const int64_t tokens = !map ? kRowBlocks / row_blocks : whole ? 64 * (16 / (int)sizeof(T)) : MapLines<T>::kTokens;
    const int64_t slab = slab_tokens(B, per_y);  // (tiles of maps have 256 tokens: fewer threads than rows)
    for (int64_t b = 0; b < B; b += slab_b) {
        const int64_t n_b = std::min(B - b, slab_b), k = b * kBlock, channels = std::min(K - k, slab_b * kBlock);
        for (int64_t m = 0; m < R.rows; m += slab) {
            const Mx4Rows P = {R.codes + m * R.stride + b * 16, R.stride, R.scales + b * R.scales_stride + m, R.scales_stride,
                               std::min(R.rows - m, slab)};
            const dim3 grid((unsigned)ceil_div64(P.rows, tokens), (unsigned)ceil_div64(n_b, per_y));
            T* p = out + m * (map ? 1 : ts) + k * (map ? ks : 1);
            if (!map && row_blocks == 16) dequantize_mx4_rows_kernel<T, 16><<<grid, kThreads, 0, s>>>(P, channels, p, ts, whole);
            else if (!map) dequantize_mx4_rows_kernel<T, kFewBlocks><<<grid, kThreads, 0, s>>>(P, channels, p, ts, whole);
            else if (whole) dequantize_mx4_whole_kernel<T><<<grid, kMapWaves * 64, 0, s>>>(P, channels, p, ks);
            else dequantize_mx4_map_kernel<T><<<grid, kMapWaves * 64, 0, s>>>(P, channels, p, ks);
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
