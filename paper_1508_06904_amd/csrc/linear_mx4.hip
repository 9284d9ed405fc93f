// A fully connected layer in 4 bits on the tokens of a map, in one launch: the codes go from the values' registers to the matrix
// instructions' operands and never travel.
//
// A lane that holds a block of 32 channels of V adjacent tokens (MapBlock) holds the operands of V matrix instructions, whose
// rows are V tokens apart: its codes and its scales are theirs as they are.  With the outputs' channels as the result's rows
// a lane gets V adjacent tokens of four channels, which are a map's stores of 16 bytes, 256 adjacent bytes for 16 lanes.
// The weights are in LDS.
//
// Bound by memory: the values in, the outputs out.
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
// The weights' rows are a multiple of 16 there, their scales block by block.
size_t weights_lds(int64_t N, int B) { return (size_t)ceil_div64(N, 16) * 16 * (pitch_of(B) + B); }

// S steps of 128 channels.
template <typename T, typename Tout, int S, bool MAP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2))) void linear_mx4_kernel(Mx4Layer L, Mx4Values X) {
    constexpr int V = Block<T>::V;
    extern __shared__ __align__(16) uint8_t lds[];
    const int B = L.B, N = (int)L.weight.rows, N16 = (N + 15) / 16 * 16, pitch = pitch_of(B);
    uint8_t* const scales = lds + N16 * pitch;
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
    for (int n = threadIdx.x; n < N16 * B; n += kThreads) {
        const int row = n / B, b = n - row * B, from = min(row, N - 1);
        *reinterpret_cast<i32x4*>(lds + row * pitch + b * 16) = *reinterpret_cast<const i32x4*>(L.weight.codes + from * L.weight.stride + b * 16);
        scales[b * N16 + row] = L.weight.scales[b * L.weight.scales_stride + from];
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
        float bias[4] = {};
        if (L.bias)
#pragma unroll
            for (int r = 0; r < 4; ++r) bias[r] = L.bias[min(n + r, N - 1)];
        if constexpr (MAP) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if (n + r >= N) continue;
                float out[V];
#pragma unroll
                for (int j = 0; j < V; ++j) out[j] = activate_nan(L.act, acc[j][r] + bias[r]);
                store_values(static_cast<Tout*>(L.out) + (n + r) * L.ldo + m, out, 0, V, L.past);
            }
        } else {
            if (n < N)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float out[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) out[r] = activate_nan(L.act, acc[j][r] + bias[r]);
                    store_values(static_cast<Tout*>(L.out) + (m + j) * L.ldo + n, out, n, N, L.past);
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

constexpr int64_t kLeastTokens = 4096;

}  // namespace

bool linear_mx4_at_once(int64_t M, int64_t N, int64_t K, bool map) {
    return map && M >= kLeastTokens && K <= 512 && weights_lds(N, (int)blocks_of(K)) <= 72 * 1024;
}

hipError_t launch_linear_mx4(const Mx4Layer& L, const Mx4Values& X, dss_dtype out_dtype, hipStream_t s) {
    // slabs of equal size but for the last, none below kLeastTokens
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
