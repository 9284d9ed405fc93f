// A fully connected layer in 4 bits on the tokens of a map, in one launch: the codes go from the values' registers to the matrix
// instructions' operands and never travel.
//
// A lane that holds a block of 32 channels of V adjacent tokens (MapBlock) holds the operands of V matrix instructions, whose
// rows are V tokens apart: its codes and its scales are theirs as they are.  With the outputs' channels as the result's rows
// a lane gets V adjacent tokens of four channels, which are a map's stores of 16 bytes, 256 adjacent bytes for 16 lanes.
// The weights are in LDS.
//
// Bound by memory: the values in, the outputs out.  1.88 million tokens of 512 channels to 128 in binary32, map in and map out:
// 1.10 ms (4.3 TB/s), and 0.96 (5.0) where the map's rows are whole lines; at a large copy's 4.85 TB/s it would be 0.99.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

// Four tokens for a lane: eight of bfloat16 would need 128 registers for their codes of 512 channels.
template <typename T>
using Block = MapBlock<T, (int)sizeof(T)>;

// A weight row's codes in LDS: 16 bytes more than it has, so that rows start in different banks.
__host__ __device__ constexpr int pitch_of(int B) { return B * 16 + 16; }
// The weights' rows are a multiple of 16 there, their scales block by block; and the bias (loaded beside the outputs' stores it
// would wait for them).
size_t weights_lds(int64_t N, int B) { return (size_t)ceil_div64(N, 16) * 16 * (pitch_of(B) + B + 4); }

// S steps of 128 channels.
template <typename T, typename Tout, int S, bool MAP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void linear_mx4_kernel(Mx4Layer L, Mx4Values X) {
    constexpr int V = Block<T>::V;
    extern __shared__ __align__(16) uint8_t lds[];
    const int B = L.B, N = (int)L.weight.rows, N16 = (N + 15) / 16 * 16, pitch = pitch_of(B);
    float* const biases = reinterpret_cast<float*>(lds + N16 * pitch);
    uint8_t* const scales = reinterpret_cast<uint8_t*>(biases + N16);
    const int lane = threadIdx.x & 63, l16 = lane & 15, q16 = lane >> 4;
    const int64_t M = L.tokens.rows, K = X.channels, ks = X.channel_stride;
    // (the last tile ends with the last token, and computes what the ones before it have over again)
    const int64_t tile = xcd_order(blockIdx.x, gridDim.x) * kWaves + (threadIdx.x >> 6);
    const int64_t m = min(tile * Block<T>::kTokens, M - Block<T>::kTokens) + l16 * V;
    i32x4 codes[S][V];
    uint32_t bytes[S];
    Block<T> v;
    auto load = [&](int s) {
        const int64_t k = (s * 4 + q16) * kBlock;
        v.load(static_cast<const T*>(X.x) + m + k * ks, ks, (int)max(min((int64_t)kBlock, K - k), (int64_t)0));
    };
    // the first values are on their way while the weights are put into LDS
    load(0);
    for (int n = threadIdx.x; n < N16; n += kThreads) biases[n] = L.bias ? L.bias[min(n, N - 1)] : 0.f;
    constexpr int U = 8;                 // of them under way
    for (int n0 = threadIdx.x; n0 < N16 * B; n0 += U * kThreads) {
        i32x4 w[U];
        uint8_t x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int n = min(n0 + u * kThreads, N16 * B - 1), from = min(n / B, N - 1);
            w[u] = *reinterpret_cast<const i32x4*>(L.weight.codes + from * L.weight.stride + (n % B) * 16);
            // (in the order in which they lie)
            x[u] = L.weight.scales[n / N16 * L.weight.scales_stride + min(n % N16, N - 1)];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int n = n0 + u * kThreads;
            if (n >= N16 * B) continue;
            *reinterpret_cast<i32x4*>(lds + n / B * pitch + (n % B) * 16) = w[u];
            scales[n] = x[u];
        }
    }
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s) load(s);
        uint32_t byte[V];
        v.scale_bytes(byte);
        bytes[s] = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            codes[s][j] = v.codes(j, byte[j]);
            bytes[s] |= byte[j] << (8 * j);
        }
    }
    __syncthreads();
    for (int n0 = 0; n0 < N; n0 += 16) {
        f32x4 acc[V] = {};
#pragma unroll
        for (int s = 0; s < S; ++s) {
            // (past the end of K the tokens' codes are zeros; the last block's weights are there)
            const int b = min(s * 4 + q16, B - 1);
            const i32x4 w = *reinterpret_cast<const i32x4*>(lds + (n0 + l16) * pitch + b * 16);
            const uint32_t w_scale = scales[b * N16 + n0 + l16];
#pragma unroll
            for (int j = 0; j < V; ++j) acc[j] = multiply_at(j, w, w_scale, codes[s][j], bytes[s], acc[j]);
        }
        const int n = n0 + q16 * 4;
        const f32x4 bias = *reinterpret_cast<const f32x4*>(biases + n);
        float out[4 * V];                // [channel][token] of a map, [token][channel] of rows
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) out[MAP ? r * V + j : j * 4 + r] = acc[j][r] + bias[r];
        activate_all(L.act, out);
        constexpr int LINES = MAP ? 4 : V, PER = MAP ? V : 4;
#pragma unroll
        for (int l = 0; l < LINES; ++l) {
            float line[PER];
#pragma unroll
            for (int i = 0; i < PER; ++i) line[i] = out[l * PER + i];
            // (a row's 16 channels are parts of lines, which only the caches put together: 64 channels to 128 outputs of 1.88 million
            // bfloat16 tokens 257 us, around the caches 552; a map's stores are whole ones, 133 us, through the caches 165)
            if constexpr (MAP) {
                if (n + l < N) store_values(static_cast<Tout*>(L.out) + (n + l) * L.ldo + m, line, 0, V, L.past);
            } else {
                if (n < N) store_values(static_cast<Tout*>(L.out) + (m + l) * L.ldo + n, line, n, N, 0);
            }
        }
    }
}

template <typename T, typename Tout, int S>
hipError_t run_linear(const Mx4Layer& L, const Mx4Values& X, hipStream_t s) {
    const size_t lds = weights_lds(L.weight.rows, L.B);
    const auto kern = L.map ? linear_mx4_kernel<T, Tout, S, true> : linear_mx4_kernel<T, Tout, S, false>;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)ceil_div64(L.tokens.rows, Block<T>::kTokens * kWaves)), kThreads, lds, s>>>(L, X);
    return hipGetLastError();
}

template <typename T, typename Tout>
hipError_t run_steps(const Mx4Layer& L, const Mx4Values& X, hipStream_t s) {
    return L.B <= 8 ? run_linear<T, Tout, 2>(L, X, s) : run_linear<T, Tout, 4>(L, X, s);
}

constexpr int64_t kLeastTokens = 256;

}  // namespace

// Where one launch is the faster one.  In microseconds for one launch and for two (GPU, outputs a binary32 map), channels to
// outputs:
//                binary32: 64-256    256-16    256-64   256-256   512-128   bfloat16: 64-256    256-64   256-256   512-128
//   1000 tokens            14/8       7/8       9/8      15/8      17/9               14/10     9/9      15/9      16/10
//   20000                  17/15      9/12     11/13     19/17     21/19              17/16    11/12     18/16     20/16
//   100000                 27/36     25/36     29/39     52/55     58/73              25/35    23/30     42/46     43/54
//   400000                135/150    95/125   117/146   201/249   238/295            129/136   74/99    168/211   156/212
// The rule takes all of them from 32768 tokens on; few outputs of few channels, where the two are about as fast on the GPU,
// for the launch and the workspace that a call then does without, from 256 on.  Two of those measured lose: 1.88 million bfloat16
// tokens of 64 channels to 256 outputs (697/645) and 1000 binary32 tokens of 256 channels to 64 (9/8; in a captured graph 8.6/7.7).
bool linear_mx4_at_once(int64_t M, int64_t N, int64_t K, bool map) {
    const bool fits = map && K <= 512 && weights_lds(N, (int)blocks_of(K)) <= 72 * 1024;
    return fits && (M >= 32768 || (M >= kLeastTokens && N <= 64 && K <= 256));
}

hipError_t launch_linear_mx4(const Mx4Layer& L, const Mx4Values& X, dss_dtype out_dtype, hipStream_t s) {
    // (slabs of equal size but for the last, none below a tile)
    const int64_t slab = ceil_div64(L.tokens.rows, ceil_div64(L.tokens.rows, (int64_t)1 << 29));
    for (int64_t m = 0; m < L.tokens.rows; m += slab) {
        Mx4Layer P = L;
        Mx4Values Y = X;
        P.tokens.rows = std::min(L.tokens.rows - m, slab);
        P.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        Y.x = static_cast<const char*>(X.x) + m * (int64_t)dtype_size(X.dtype);
        hipError_t e;
        if (X.dtype == DSS_BF16)
            e = out_dtype == DSS_BF16 ? run_steps<uint16_t, uint16_t>(P, Y, s) : run_steps<uint16_t, float>(P, Y, s);
        else
            e = out_dtype == DSS_BF16 ? run_steps<float, uint16_t>(P, Y, s) : run_steps<float, float>(P, Y, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace dss
