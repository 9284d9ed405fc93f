// Products of a few 8-bit tokens with 8-bit weights: a server's single tokens.
//
// At most 16 GT tokens: bound by the weights' bytes, which are read once.  A
// workgroup takes 16 outputs; its waves divide K in turns of kSlab bytes, straight from
// memory to matrix operands (any address), and add their sums through LDS.  With few
// outputs a workgroup takes fewer of them, down to two, so that all 256 units read.
//
// One window through 9216 x 512 with the coding: 8.4 us, of which 4.7 MB of weights at 5 TB/s are
// 0.9: a chain of latencies (the values, their largest, the codes, up to five slabs of weights
// that each wave fetches in turn, the sums).  32 tokens through 4096 x 4096: 9.1 us.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

constexpr int kSlab = 256;
constexpr int kFewWaves = 8;

// Where the tokens come from: codes in memory (Code = int8_t), or values that the
// workgroup codes itself into LDS (float, uint16_t), which costs every workgroup a
// reading of all tokens and saves a launch and the codes' way through memory.
constexpr int kFewValues = 16384;        // values that a workgroup codes at most (their tokens as a power of two)

// Codes and scales of the M <= 16 tokens, in LDS: codes[m * pitch + k], zeros from K to the pitch.
template <typename T>
__device__ void code_few(const Values& V, int M, int K, int pitch, int8_t* codes, float* scales, uint32_t* tops) {
    constexpr int E = Chunk<T>::E, THREADS = kFewWaves * 64, CH = 2 * kFewValues / THREADS / E;
    // THREADS / 2^b lanes for each token
    const int b = M <= 1 ? 0 : 32 - __clz(M - 1);
    const int lanes = THREADS >> b, m = threadIdx.x / lanes, lane = threadIdx.x % lanes;
    if (threadIdx.x < 16) tops[threadIdx.x] = 0;
    __syncthreads();
    Chunk<T> c[CH];
    uint32_t top = 0;
    if (m < M) {
        const T* row = static_cast<const T*>(V.x) + m * V.token_stride;
        if (V.channel_stride == 1) {
            load_row(c, row, lane, lanes, K);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int k = 0; k < E; ++k) {
                    const int at = (i * lanes + lane) * E + k;
                    if (at < K) c[i].set(k, row[at * V.channel_stride]);
                }
        }
#pragma unroll
        for (int i = 0; i < CH; ++i) top = raise(top, c[i]);
    }
    top = top_bits<T>(top);
#pragma unroll
    for (int d = 16; d; d >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, d));
    if ((threadIdx.x & 31) == 0 && m < M) atomicMax(&tops[m], top);   // (a maximum has no order)
    __syncthreads();
    if (m < M) {
        const Coder coder(scale_of(tops[m]));
        if (lane == 0) scales[m] = coder.scale;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = (i * lanes + lane) * E;
            if (at < pitch) store_codes(codes + m * pitch + at, c[i], coder, E);
        }
    }
    __syncthreads();
}

// The codes' row length in LDS: whole slabs and 16 bytes, so that tokens start in different banks.
__host__ __device__ constexpr int few_pitch(int K) { return (K + kSlab - 1) / kSlab * kSlab + 16; }

// ODD: weights or codes that start inside words.
template <typename Code, typename Tout, int GT, bool MAP, bool ODD>
__global__ __launch_bounds__(kFewWaves * 64) void matmul_few_kernel(Layer L, Values V, int R) {
    constexpr bool kCodes = sizeof(Code) == 1;
    __shared__ i32x4 part[kFewWaves][GT][64];
    __shared__ float own_scales[16];
    __shared__ uint32_t tops[16];
    extern __shared__ __align__(16) int8_t own_codes[];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, q16 = lane >> 4;
    const int8_t* t[GT];
    const int K = L.K;
    constexpr int H = kSlab / 64;
    auto weights = [&](int tile) { return L.weight + (int64_t)min(tile * R + min(l16, R - 1), L.N - 1) * L.weight_stride; };
    const int8_t* const w_end = L.weight + (L.N - 1) * L.weight_stride + K;
    const int8_t* const c_end = L.codes + (L.M - 1) * L.codes_stride + K;
    auto fetch = [&](const int8_t* row, int k0, i32x4* to, const int8_t* begin, const int8_t* end) {
#pragma unroll
        for (int h = 0; h < H; ++h) {
            const int8_t* from = row + k0 + h * 64 + q16 * 16;
            if constexpr (ODD) to[h] = load_any(from, begin, end);
            else __builtin_memcpy(&to[h], from, 16);
        }
    };
    auto multiply = [](i32x4 u, i32x4 v, i32x4 c) {
        return MAP ? __builtin_amdgcn_mfma_i32_16x16x64_i8(v, u, c, 0, 0, 0)
                   : __builtin_amdgcn_mfma_i32_16x16x64_i8(u, v, c, 0, 0, 0);
    };
    i32x4 a[H], b[GT][H];
    // the first weights are on their way while the tokens are coded
    const int8_t* w = weights(blockIdx.x);
    const int k_first = wave * kSlab, k_whole = K / kSlab * kSlab;
    if (!kCodes && k_first < k_whole) fetch(w, k_first, a, L.weight, w_end);
    if constexpr (kCodes) {
#pragma unroll
        for (int g = 0; g < GT; ++g) t[g] = L.codes + min((int64_t)(g * 16 + l16), L.M - 1) * L.codes_stride;
    } else {
        code_few<Code>(V, (int)L.M, K, few_pitch(K), own_codes, own_scales, tops);
        t[0] = own_codes + min(l16, (int)L.M - 1) * few_pitch(K);
        L.scales = own_scales;
    }
    const int tiles = (L.N + R - 1) / R;
    for (int tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        if (tile != (int)blockIdx.x) {
            w = weights(tile);
            __syncthreads();             // the sums of the last tile have been read
        }
        i32x4 acc[GT] = {};
        auto fetch_tokens = [&](int k0) {
#pragma unroll
            for (int g = 0; g < GT; ++g) {
                if constexpr (kCodes) {
                    fetch(t[g], k0, b[g], L.codes, c_end);
                } else {
#pragma unroll
                    for (int h = 0; h < H; ++h) b[g][h] = *reinterpret_cast<const i32x4*>(t[g] + k0 + h * 64 + q16 * 16);
                }
            }
        };
        for (int k0 = k_first; k0 < k_whole; k0 += kFewWaves * kSlab) {
            if (kCodes || k0 != k_first || tile != (int)blockIdx.x) fetch(w, k0, a, L.weight, w_end);
            fetch_tokens(k0);
#pragma unroll
            for (int h = 0; h < H; ++h)
#pragma unroll
                for (int g = 0; g < GT; ++g) acc[g] = multiply(a[h], b[g][h], acc[g]);
        }
        // the slab that K ends in, if it ends in one
        if (k_whole < K && k_whole / kSlab % kFewWaves == wave) {
#pragma unroll 1
            for (int k0 = k_whole; k0 < K; k0 += 64) {
                const int k = k0 + q16 * 16;
                const i32x4 u = load_unit(w, k, K);
#pragma unroll
                for (int g = 0; g < GT; ++g) {
                    const i32x4 v = kCodes ? load_unit(t[g], k, K) : *reinterpret_cast<const i32x4*>(t[g] + k);
                    acc[g] = multiply(u, v, acc[g]);
                }
            }
        }
#pragma unroll
        for (int g = 0; g < GT; ++g) part[wave][g][lane] = acc[g];
        __syncthreads();
        if (wave >= GT) continue;
        i32x4 sum = part[0][wave][lane];
#pragma unroll
        for (int v = 1; v < kFewWaves; ++v) sum += part[v][wave][lane];
        // MAP: the lane has output n0 + l16 of four tokens; rows: four outputs of token l16
        const int n0 = tile * R, n_end = min(n0 + R, L.N);
        const int64_t i = MAP ? n0 + l16 : wave * 16 + l16, j = MAP ? wave * 16 + q16 * 4 : n0 + q16 * 4;
        const int64_t I = MAP ? n_end : L.M, J = MAP ? L.M : n_end;
        if (i < I && j < J) store_outputs<Tout, MAP>(L, i, j, J, &sum, side_i<MAP>(L, i), side_j<MAP>(L, j));
    }
}

template <typename Code, typename Tout, int GT>
hipError_t run_few(const Layer& L, const Values& V, hipStream_t s) {
    static_assert(GT <= kFewWaves, "a wave adds up one group of tokens");
    int R = 16;
    while (R > 2 && ceil_div64(L.N, R) < 256) R /= 2;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div64(L.N, R), sizeof(Code) == 1 ? 4096 : 256));
    const size_t lds = sizeof(Code) == 1 ? 0 : (size_t)L.M * few_pitch(L.K);
    auto words = [](const int8_t* p, int64_t stride, int64_t rows) {
        return (uintptr_t)p % 4 == 0 && (stride % 4 == 0 || rows == 1);
    };
    const bool odd = !words(L.weight, L.weight_stride, L.N) || (sizeof(Code) == 1 && !words(L.codes, L.codes_stride, L.M));
    const auto kern = L.map ? (odd ? matmul_few_kernel<Code, Tout, GT, true, true> : matmul_few_kernel<Code, Tout, GT, true, false>)
                            : (odd ? matmul_few_kernel<Code, Tout, GT, false, true> : matmul_few_kernel<Code, Tout, GT, false, false>);
    kern<<<grid, kFewWaves * 64, lds, s>>>(L, V, R);
    return hipGetLastError();
}

template <typename Code, typename Tout>
hipError_t run_groups(const Layer& L, const Values& V, hipStream_t s) {
    if constexpr (sizeof(Code) == 1) {
        if (L.M > 16) return run_few<Code, Tout, 2>(L, V, s);
    }
    return run_few<Code, Tout, 1>(L, V, s);
}

}  // namespace

// Up to 32 tokens.  Codes in hand, here and on tiles, us on the GPU, of 1, 13 and 32 tokens
// through 4096 x 4096: 6.7/10.7, 7.0/10.7, 9.1/11.5; 9216 x 8192: 16/29, 22/29, 33/30; 4096 x
// 16384: 17/21, 20/21, 29/22; 1024 x 32768: 11.0/10.2, 13.2/10.9, 19.0/12.8.  The tiles gain
// with the outputs (whose tiles fill the units) and with the tokens, and lose where weights
// would be copied for them; K, and with it the weights' size, does not decide.  A width of
// 8192 alone is a coarse rule: up to 13 tokens of 4096 x 16384 are faster here, 32 of 9216 x
// 8192 on tiles.
bool few_tokens(int64_t M, int N, int K) { return M <= 32 && (N <= 8192 || K % 16 != 0); }

hipError_t launch_matmul_few(const Layer& L, dss_dtype out_dtype, hipStream_t s) {
    return out_dtype == DSS_BF16 ? run_groups<int8_t, uint16_t>(L, Values{}, s) : run_groups<int8_t, float>(L, Values{}, s);
}

// Tokens of 1, 2 and 4 that the kernel codes itself, and coded by a launch before, us on the GPU:
// 9216 x 512 8.4/10.7 (one token); 4096 x 4096 9.0/9.8, 9.7/9.9, 10.7/10.0; 4096 x 16384 20.9/24.1,
// 22.0/24.6, 23.3/24.6; 9216 x 8192 (one) 22.4/21.6; 1024 x 32768 16.9/13.3, 17.2/13.4, 17.7/13.6:
// the outputs are not in the rule, though layers of many outputs and few channels would be
// better coded first.
bool codes_itself(int64_t M, int K) {
    if (M > 16) return false;
    int p = 1;
    while (p < M) p *= 2;
    return (int64_t)p * K <= kFewValues;
}

hipError_t launch_linear_few(const Layer& L, const Values& V, dss_dtype out_dtype, hipStream_t s) {
    if (V.dtype == DSS_BF16)
        return out_dtype == DSS_BF16 ? run_groups<uint16_t, uint16_t>(L, V, s) : run_groups<uint16_t, float>(L, V, s);
    return out_dtype == DSS_BF16 ? run_groups<float, uint16_t>(L, V, s) : run_groups<float, float>(L, V, s);
}

}  // namespace dss
