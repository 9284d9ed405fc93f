// A fully connected layer on the tokens of a map in one launch: a workgroup codes its
// tokens into LDS and multiplies them with all of the weights from there.
//
// The tokens' values are read once, and their codes never travel: in two launches
// they are written to and read back from memory, a byte each way beside the 4 (or
// 2) of a value.  In exchange every workgroup reads all weights, from L2; that
// stays below the codes' traffic while the weights are few (linear_in_tiles).
// Bound by memory: the values in, the outputs out.  1.88 million tokens of 512 channels to 128 in
// binary32, map in and map out: 1.13 to 1.20 ms, 4.0 to 4.2 TB/s; at a large copy's 5.07 TB/s
// it would be 0.95.  The difference is the outputs' rows, which end inside lines there.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

constexpr int kMaxChannels = kMapWaves * 64;       // of a token in registers, and in LDS

// A token's codes in LDS: whole matrix operands of 64, and 16 bytes more, so that tokens start in different banks.
__host__ __device__ constexpr int tile_pitch(int K) { return (K + 63) / 64 * 64 + 16; }

// A workgroup's LDS: its tokens' codes and scales, and 64 words for each wave's largest values.  All of it is
// in the launch's own size, whose opt-in above 64 KB knows of no other.
size_t tile_lds(int tokens, int K, int waves) { return (size_t)tokens * (tile_pitch(K) + 4) + waves * 256; }

// Codes and scales of the tokens of a map from x on: tiles beside each other, `waves` waves for each.
template <typename T>
__device__ __forceinline__ void code_map(const T* x, int64_t channel_stride, int K, int waves, int pitch, int8_t* codes,
                                         float* scales, uint32_t* tops) {
    using Tile = MapTile<T>;
    const int wave = threadIdx.x >> 6, group = wave / waves, k = (wave - group * waves) * 64 + ((threadIdx.x >> 4) & 3) * 16;
    const int t = group * Tile::kTokens + (threadIdx.x & 15) * Tile::V;
    Tile tile;
    uint32_t top[4] = {};
    tile.load(x + group * Tile::kTokens, channel_stride, k, K);
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

// `tokens` tokens for each workgroup; the last one's end with the last token, and
// it leaves out what the one before it has.
template <typename T, typename Tout, bool MAP>
__global__ __launch_bounds__(kMapWaves * 64) void linear_tile_kernel(Layer L, Values V, int tokens, int waves) {
    extern __shared__ __align__(16) int8_t lds[];
    const int K = L.K, pitch = tile_pitch(K);
    float* scales = reinterpret_cast<float*>(lds + tokens * pitch);
    const int64_t tile0 = xcd_order(blockIdx.x, gridDim.x) * tokens, m0 = min(tile0, L.M - tokens);
    const int first = (int)(tile0 - m0);
    code_map(static_cast<const T*>(V.x) + m0, V.channel_stride, K, waves, pitch, lds, scales,
             reinterpret_cast<uint32_t*>(scales + tokens));
    __syncthreads();

    // 16 outputs of 64 tokens at a time for a wave
    const int lane = threadIdx.x & 63, l16 = lane & 15, q16 = lane >> 4;
    const int quarters = tokens / 64, items = (L.N + 15) / 16 * quarters;
    L.scales = scales;
    L.M = tokens;
    L.out = static_cast<Tout*>(L.out) + m0 * (MAP ? 1 : L.ldo);
    for (int item = threadIdx.x >> 6; item < items; item += blockDim.x >> 6) {
        const int n0 = item / quarters * 16, t0 = (item - item / quarters * quarters) * 64;
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
            if (i >= I || j >= J || (!MAP && i < first)) continue;
            store_outputs<Tout, MAP>(L, i, j, J, &acc[g], p[g], q[g], MAP ? first : 0);
        }
    }
}

template <typename T, typename Tout>
hipError_t run_linear(const Layer& L, const Values& V, hipStream_t s) {
    const int waves = (L.K + 63) / 64, groups = std::max(1, 8 / waves), tokens = groups * MapTile<T>::kTokens;
    const size_t lds = tile_lds(tokens, L.K, waves * groups);
    const auto kern = L.map ? linear_tile_kernel<T, Tout, true> : linear_tile_kernel<T, Tout, false>;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)ceil_div64(L.M, tokens)), waves * groups * 64, lds, s>>>(L, V, tokens, waves);
    return hipGetLastError();
}

constexpr int64_t kLeastTokens = 4096;

}  // namespace

// Where one launch is the faster one.  In microseconds for one launch and for two (GPU, outputs
// as a map), channels to outputs:
//                binary32: 256-64   512-128   256-128   512-256   bfloat16: 256-64   512-128   256-128   512-256
//   1000 tokens            9/10     11/14     12/10     15/14               14/13    16/16     19/13     24/17
//   4096                  10/12     11/14     13/12     15/15               15/14    18/17     20/14     25/18
//   20000                 12/16     21/27     16/18     28/33               16/17    20/23     22/18     30/30
//   100000                39/49     73/92     51/58     99/103              31/41    61/78     40/50     71/86
//   400000               124/159   264/331   160/191   332/419              92/117  187/257   108/142   273/353
// 1024 channels to 128: 43/45, 167/168, 605/609 and 30/36, 133/137, 417/473 for the last three.
// The rule takes the two leftmost columns and 1024-128 in both types, from 4096 tokens on:
// there bfloat16 still loses one microsecond, binary32 gains from 256 tokens on.  The wider layers,
// which gain from 20000 (binary32) and 100000 (bfloat16) tokens on, are left to two launches.
// Weights at odd addresses are read here at the price of a tenth (100000 tokens, 512-128: 76 us
// for 69 in binary32, 66 for 57 in bfloat16), which two launches (89, 73) do not win back.
// Rows of values (the channels adjacent) gain less than a tenth and are always coded first.
bool linear_in_tiles(int64_t M, int N, int K, bool map) {
    return map && M >= kLeastTokens && K <= kMaxChannels && ((K >= 512 && N <= 128) || (K >= 256 && N <= 64));
}

hipError_t launch_linear_tiles(const Layer& L, const Values& V, dss_dtype out_dtype, hipStream_t s) {
    // slabs of equal size but for the last, none below kLeastTokens
    const int64_t slabs = ceil_div64(L.M, kSlabTokens), slab = ceil_div64(L.M, slabs);
    for (int64_t m = 0; m < L.M; m += slab) {
        Layer S = L;
        Values W = V;
        S.M = std::min(L.M - m, slab);
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        W.x = static_cast<const char*>(V.x) + m * (int64_t)dtype_size(V.dtype);
        hipError_t e;
        if (V.dtype == DSS_BF16)
            e = out_dtype == DSS_BF16 ? run_linear<uint16_t, uint16_t>(S, W, s) : run_linear<uint16_t, float>(S, W, s);
        else
            e = out_dtype == DSS_BF16 ? run_linear<float, uint16_t>(S, W, s) : run_linear<float, float>(S, W, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace dss
