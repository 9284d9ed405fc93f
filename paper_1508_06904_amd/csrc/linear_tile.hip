// A fully connected layer on many tokens in one launch: a workgroup codes its tokens
// into LDS and multiplies them with all of the weights from there.
//
// The tokens' values are read once, and their codes never travel: in two launches
// they are written to and read back from memory, a byte each way beside the 4 (or
// 2) of a value.  In exchange every workgroup reads all weights, from L2; that
// stays below the codes' traffic while the weights are few (linear_in_tiles).
// Bound by memory: the values in, the outputs out.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

constexpr int kMaxChannels = 1024;       // of a token in LDS
constexpr int kRowTokens = 64;           // tokens of a workgroup, rows
constexpr int kRowWaves = 8;

// A token's codes in LDS: whole matrix operands of 64, and 16 bytes more, so that tokens start in different banks.
__host__ __device__ constexpr int tile_pitch(int K) { return (K + 63) / 64 * 64 + 16; }

// Codes and scales of the tokens of a map from x on: `groups` tiles beside each other, `waves` waves for each.
template <typename T>
__device__ __forceinline__ void code_map(const T* x, int64_t channel_stride, int64_t left, int K, int waves, int pitch,
                                         int8_t* codes, float* scales) {
    using Tile = MapTile<T>;
    __shared__ uint32_t tops[kMapWaves * 64];
    const int wave = threadIdx.x >> 6, group = wave / waves, k = (wave - group * waves) * 64 + ((threadIdx.x >> 4) & 3) * 16;
    const int t0 = group * Tile::kTokens, t = t0 + (threadIdx.x & 15) * Tile::V;
    Tile tile;
    uint32_t top[4] = {};
    tile.load(x + t0, channel_stride, (int)max((int64_t)0, min(left - t0, (int64_t)Tile::kTokens)), k, K);
    tile.raise_into(top);
    Tile::meet(top, tops, group * waves, waves);
#pragma unroll
    for (int j = 0; j < Tile::V; ++j) {
        const Coder coder(scale_of(Tile::bits(top, j)));
        if (k == 0) scales[t + j] = coder.scale;
        uint32_t w[4];
        tile.codes(j, coder, w);
        *reinterpret_cast<i32x4*>(codes + (t + j) * pitch + k) = __builtin_bit_cast(i32x4, w);
    }
}

// The same of kRowTokens rows: each wave takes an eighth of them, kTogether at a time.
template <typename T>
__device__ __forceinline__ void code_rows(const T* x, int64_t token_stride, int64_t left, int K, int pitch,
                                          int8_t* codes, float* scales) {
    constexpr int E = Chunk<T>::E, CH = kMaxChannels / 64 / E, kTogether = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
    for (int m = wave * (kRowTokens / kRowWaves); m < (wave + 1) * (kRowTokens / kRowWaves); m += kTogether) {
        Chunk<T> c[kTogether][CH];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) load_row(c[u], x + min((int64_t)(m + u), left - 1) * token_stride, lane, 64, K);
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < CH; ++i) top = raise(top, c[u][i]);
            top = top_bits<T>(top);
#pragma unroll
            for (int d = 32; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
            const Coder coder(scale_of(top));
            if (lane == 0) scales[m + u] = coder.scale;
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int at = (i * 64 + lane) * E;
                if (at < pitch - 16) store_codes(codes + (m + u) * pitch + at, c[u][i], coder, E);
            }
        }
    }
}

template <typename T, typename Tout, bool ROWS, bool MAP>
__global__ __launch_bounds__(1024) void linear_tile_kernel(Layer L, Values V, int tokens, int waves) {
    extern __shared__ __align__(16) int8_t lds[];
    const int K = L.K, pitch = tile_pitch(K);
    float* scales = reinterpret_cast<float*>(lds + tokens * pitch);
    const int64_t m0 = xcd_order(blockIdx.x, gridDim.x) * tokens, left = L.M - m0;
    if constexpr (ROWS)
        code_rows(static_cast<const T*>(V.x) + m0 * V.token_stride, V.token_stride, left, K, pitch, lds, scales);
    else
        code_map(static_cast<const T*>(V.x) + m0, V.channel_stride, left, K, waves, pitch, lds, scales);
    __syncthreads();

    // 16 outputs of 64 tokens at a time for a wave
    const int lane = threadIdx.x & 63, l16 = lane & 15, q16 = lane >> 4;
    const int quarters = tokens / 64, items = (L.N + 15) / 16 * quarters;
    L.scales = scales;
    L.M = min(left, (int64_t)tokens);
    L.out = static_cast<Tout*>(L.out) + m0 * (MAP ? 1 : L.ldo);
    for (int item = threadIdx.x >> 6; item < items; item += blockDim.x >> 6) {
        const int n0 = item / quarters * 16, t0 = (item - item / quarters * quarters) * 64;
        if (t0 >= L.M) continue;
        const int8_t* w = L.weight + (int64_t)min(n0 + l16, L.N - 1) * L.weight_stride;
        const int8_t* t = lds + (t0 + l16) * pitch + q16 * 16;
        i32x4 acc[4] = {};
        auto step = [&](int k0, i32x4 a) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const i32x4 b = *reinterpret_cast<const i32x4*>(t + g * 16 * pitch + k0);
                acc[g] = MAP ? __builtin_amdgcn_mfma_i32_16x16x64_i8(b, a, acc[g], 0, 0, 0)
                             : __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, acc[g], 0, 0, 0);
            }
        };
        int k0 = 0;
        for (; k0 + 256 <= K; k0 += 256) {
            i32x4 a[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) __builtin_memcpy(&a[h], w + k0 + h * 64 + q16 * 16, 16);
#pragma unroll
            for (int h = 0; h < 4; ++h) step(k0 + h * 64, a[h]);
        }
        for (; k0 < K; k0 += 64) step(k0, load_unit(w, k0 + q16 * 16, K));
        const int64_t I = MAP ? L.N : L.M, J = MAP ? L.M : L.N;
        Side1 p[4];
        SideN<4> q[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            p[g] = side_i<MAP>(L, MAP ? n0 + l16 : t0 + g * 16 + l16);
            q[g] = side_j<MAP>(L, MAP ? t0 + g * 16 + q16 * 4 : n0 + q16 * 4);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int64_t i = MAP ? n0 + l16 : t0 + g * 16 + l16, j = MAP ? t0 + g * 16 + q16 * 4 : n0 + q16 * 4;
            if (i < I && j < J) store_outputs<Tout, MAP>(L, i, j, J, &acc[g], p[g], q[g]);
        }
    }
}

template <typename T, typename Tout, bool ROWS, bool MAP>
hipError_t run_linear(const Layer& L, const Values& V, hipStream_t s) {
    int tokens = kRowTokens, waves = kRowWaves, groups = 1;
    if (!ROWS) {
        waves = (L.K + 63) / 64;
        groups = std::max(1, 8 / waves);
        tokens = groups * MapTile<T>::kTokens;
    }
    const size_t lds = (size_t)tokens * (tile_pitch(L.K) + 4);
    const auto kern = linear_tile_kernel<T, Tout, ROWS, MAP>;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)ceil_div64(L.M, tokens)), waves * groups * 64, lds, s>>>(L, V, tokens, waves);
    return hipGetLastError();
}

template <typename T, typename Tout>
hipError_t run_layouts(const Layer& L, const Values& V, hipStream_t s) {
    if (V.channel_stride == 1 || L.K == 1)
        return L.map ? run_linear<T, Tout, true, true>(L, V, s) : run_linear<T, Tout, true, false>(L, V, s);
    return L.map ? run_linear<T, Tout, false, true>(L, V, s) : run_linear<T, Tout, false, false>(L, V, s);
}

}  // namespace

bool linear_in_tiles(int64_t M, int N, int K) { return !few_tokens(M, N) && K <= kMaxChannels && N <= 256; }

hipError_t launch_linear_tiles(const Layer& L, const Values& V, dss_dtype out_dtype, hipStream_t s) {
    for (int64_t m = 0; m < L.M; m += kSlabTokens) {
        Layer S = L;
        Values W = V;
        S.M = std::min(L.M - m, kSlabTokens);
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        W.x = static_cast<const char*>(V.x) + m * V.token_stride * (int64_t)dtype_size(V.dtype);
        hipError_t e;
        if (V.dtype == DSS_BF16)
            e = out_dtype == DSS_BF16 ? run_layouts<uint16_t, uint16_t>(S, W, s) : run_layouts<uint16_t, float>(S, W, s);
        else
            e = out_dtype == DSS_BF16 ? run_layouts<float, uint16_t>(S, W, s) : run_layouts<float, float>(S, W, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace dss
