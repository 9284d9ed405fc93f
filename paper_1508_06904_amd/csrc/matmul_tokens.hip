// Products of 8-bit tokens with 8-bit weights:
//   y[m][n] = act(scale[m] * weight_scale[n] * sum_k code[m][k] * weight[n][k] + bias[n]).
//
// The sums are exact: v_mfma_i32_16x16x64_i8 over 32-bit integers, whose range K
// <= 131071 keeps (128 * 128 * 131071 < 2^31).  Integers add in any order to the same bits,
// so tiles, and the division of K, are free to follow the sizes.
//
// D[i][j] = sum_k P[i][k] Q[j][k] with the output's adjacent axis as j: for rows
// P are the tokens and Q the weights, for dense maps the other way round.  In the
// matrix instruction Q's rows are the result's rows, so that a lane holds four
// adjacent outputs.
#include <algorithm>
#include <cmath>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

using i32x4 = __attribute__((ext_vector_type(4))) int;

struct Layer {
    const int8_t* codes;
    int64_t codes_stride;
    const float* scales;
    int64_t M;
    const int8_t* weight;
    int64_t weight_stride;
    const float* weight_scales;
    int N, K;
    const float* bias;
    int act;
    void* out;
    int64_t ldo;                         // the output's stride that is not 1
    int map;                             // out is [N][M], not [M][N]
};

// A NaN stays one (fmaxf would make it 0).
__device__ __forceinline__ float activate_nan(int act, float v) {
    if (act == DSS_ACT_RELU) return v < 0.f ? 0.f : v;
    if (act == DSS_ACT_TANH) return tanhf(v);
    return v;
}

__device__ __forceinline__ float output_of(int sum, float wscale, float scale, float bias, int act) {
    return activate_nan(act, (float)sum * wscale * scale + bias);
}

// D's operands and extents.
struct Sides {
    const int8_t *P, *Q;
    int64_t ps, qs, I, J;
};
__host__ __device__ __forceinline__ Sides sides_of(const Layer& L) {
    if (L.map) return {L.weight, L.codes, L.weight_stride, L.codes_stride, L.N, L.M};
    return {L.codes, L.weight, L.codes_stride, L.weight_stride, L.M, L.N};
}

// Four adjacent outputs D[i][j .. j+3] of a layer, those from J on left out.
template <typename Tout>
__device__ __forceinline__ void store_outputs(const Layer& L, int64_t i, int64_t j, int64_t J, i32x4 sum) {
    Tout* p = static_cast<Tout*>(L.out) + i * L.ldo + j;
    struct Four {
        Tout v[4];
    } r;
    const int n = (int)min(J - j, (int64_t)4);
    if (L.map) {
        const float ws = L.weight_scales[i], b = L.bias ? L.bias[i] : 0.f;
#pragma unroll
        for (int k = 0; k < 4; ++k) store_elem(&r.v[k], output_of(sum[k], ws, k < n ? L.scales[j + k] : 0.f, b, L.act));
    } else {
        const float s = L.scales[i];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            store_elem(&r.v[k], output_of(sum[k], k < n ? L.weight_scales[j + k] : 0.f, s,
                                          L.bias && k < n ? L.bias[j + k] : 0.f, L.act));
    }
    if (n == 4) {
        __builtin_memcpy(p, &r, sizeof r);
    } else {
#pragma unroll
        for (int k = 0; k < 3; ++k)
            if (k < n) p[k] = r.v[k];
    }
}

// ------------------------------------------------------------------ tiles
// BI x BJ outputs for WI x WJ waves; kStep bytes of K at a time through two LDS
// buffers, the next step's bytes on their way while this one's are multiplied.  A
// row of a buffer is 8 units of 16 bytes; row r keeps unit u at place u ^ (r & 7),
// so that the 8 rows that a matrix operand's read takes at once lie in different
// banks.
//
// DMA: global memory to LDS without a stop in registers; rows have to start at
// 16-byte units, and K ends at one.  Otherwise through registers, from any address.
constexpr int kStep = 128;
constexpr int kUnits = kStep / 16;

// 16 zero bytes: the source of the units past the end of K.
__device__ __attribute__((aligned(16))) const unsigned int g_zero16[4] = {0u, 0u, 0u, 0u};

typedef __attribute__((address_space(3))) void lds_void;

// Bytes k .. k+15 of a row of K bytes, zeros past its end; nothing past the end is read.
__device__ __forceinline__ i32x4 load_unit(const int8_t* row, int k, int K) {
    i32x4 v = {};
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K) {
        if (K >= 16) {
            unsigned __int128 w;
            __builtin_memcpy(&w, row + K - 16, 16);
            w >>= 8 * (k + 16 - K);
            __builtin_memcpy(&v, &w, 16);
        } else {
            for (int b = 0; b < K - k; ++b) v[b >> 2] |= (int)(uint8_t)row[k + b] << (8 * (b & 3));
        }
    }
    return v;
}

// Workgroups are handed to the 8 XCDs in turn: the id of the tile that makes the
// tiles of one XCD (and of its L2) neighbours.
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t n) {
    const int64_t x = b & 7, q = n >> 3, r = n & 7;
    return x * q + min(x, r) + (b >> 3);
}

template <typename Tout, int BI, int BJ, int WI, int WJ, bool DMA>
__global__ __launch_bounds__(WI* WJ * 64) void matmul_tile_kernel(Layer L, int tiles_i, int tiles_j) {
    constexpr int NW = WI * WJ, THREADS = NW * 64;
    constexpr int TI = BI / WI / 16, TJ = BJ / WJ / 16;
    constexpr int LP = BI * kUnits / THREADS, LQ = BJ * kUnits / THREADS;   // units of each thread and step
    static_assert(LP * THREADS == BI * kUnits && LQ * THREADS == BJ * kUnits && THREADS % 64 == 0, "tile");
    constexpr int BUF = (BI + BJ) * kStep;
    extern __shared__ __align__(16) char lds[];
    const Sides S = sides_of(L);
    // tiles in strips of 8 along i: a strip's tiles share their rows of Q in cache
    const int64_t id = xcd_order(blockIdx.x, (int64_t)tiles_i * tiles_j);
    const int64_t strip = id / ((int64_t)8 * tiles_j), in_strip = id - strip * 8 * tiles_j;
    const int rows = min(8, tiles_i - (int)strip * 8);
    const int64_t i0 = (strip * 8 + in_strip % rows) * BI, j0 = in_strip / rows * BJ;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wi = wave / WJ, wj = wave % WJ;

    // the thread's units: rows row0 + n * (THREADS / 8), and one place in each of them
    const int row0 = tid >> 3, unit = (tid & 7) ^ (row0 & 7);
    const int8_t *src_p[LP], *src_q[LQ];
#pragma unroll
    for (int n = 0; n < LP; ++n) src_p[n] = S.P + min(i0 + row0 + n * (THREADS / 8), S.I - 1) * S.ps;
#pragma unroll
    for (int n = 0; n < LQ; ++n) src_q[n] = S.Q + min(j0 + row0 + n * (THREADS / 8), S.J - 1) * S.qs;

    const int K = L.K, steps = (K + kStep - 1) / kStep;
    i32x4 acc[TI][TJ] = {};
    i32x4 rp[DMA ? 1 : LP], rq[DMA ? 1 : LQ];

    auto fetch = [&](int s) {
        const int k = s * kStep + unit * 16;
        if constexpr (DMA) {
            char* to = lds + (s & 1) * BUF + wave * 1024;
            const bool in = k < K;
#pragma unroll
            for (int n = 0; n < LP; ++n)
                __builtin_amdgcn_global_load_lds(in ? (const void*)(src_p[n] + k) : (const void*)g_zero16,
                                                 (lds_void*)(to + n * THREADS * 16), 16, 0, 0);
#pragma unroll
            for (int n = 0; n < LQ; ++n)
                __builtin_amdgcn_global_load_lds(in ? (const void*)(src_q[n] + k) : (const void*)g_zero16,
                                                 (lds_void*)(to + BI * kStep + n * THREADS * 16), 16, 0, 0);
        } else {
#pragma unroll
            for (int n = 0; n < LP; ++n) rp[n] = load_unit(src_p[n], k, K);
#pragma unroll
            for (int n = 0; n < LQ; ++n) rq[n] = load_unit(src_q[n], k, K);
        }
    };
    auto put = [&](int s) {
        if constexpr (!DMA) {
            char* to = lds + (s & 1) * BUF + tid * 16;
#pragma unroll
            for (int n = 0; n < LP; ++n) *reinterpret_cast<i32x4*>(to + n * THREADS * 16) = rp[n];
#pragma unroll
            for (int n = 0; n < LQ; ++n) *reinterpret_cast<i32x4*>(to + BI * kStep + n * THREADS * 16) = rq[n];
        }
    };

    fetch(0);
    put(0);
    __syncthreads();
    const int l16 = lane & 15, q16 = lane >> 4;
    for (int s = 0; s < steps; ++s) {
        if (s + 1 < steps) fetch(s + 1);
        const char* bp = lds + (s & 1) * BUF + (wi * TI * 16 + l16) * kStep;
        const char* bq = lds + (s & 1) * BUF + BI * kStep + (wj * TJ * 16 + l16) * kStep;
#pragma unroll
        for (int h = 0; h < kStep / 64; ++h) {
            const int place = ((h * 4 + q16) ^ (l16 & 7)) * 16;
            i32x4 p[TI], q[TJ];
#pragma unroll
            for (int t = 0; t < TJ; ++t) q[t] = *reinterpret_cast<const i32x4*>(bq + t * 16 * kStep + place);
#pragma unroll
            for (int t = 0; t < TI; ++t) p[t] = *reinterpret_cast<const i32x4*>(bp + t * 16 * kStep + place);
#pragma unroll
            for (int a = 0; a < TI; ++a)
#pragma unroll
                for (int b = 0; b < TJ; ++b) acc[a][b] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[b], p[a], acc[a][b], 0, 0, 0);
        }
        if (s + 1 < steps) put(s + 1);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < TI; ++a) {
        const int64_t i = i0 + (wi * TI + a) * 16 + l16;
#pragma unroll
        for (int b = 0; b < TJ; ++b) {
            const int64_t j = j0 + (wj * TJ + b) * 16 + q16 * 4;
            if (i < S.I && j < S.J) store_outputs<Tout>(L, i, j, S.J, acc[a][b]);
        }
    }
}

template <typename Tout, int BI, int BJ, int WI, int WJ, bool DMA>
hipError_t run_tile(const Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int64_t ti = ceil_div64(S.I, BI), tj = ceil_div64(S.J, BJ);
    const auto kern = matmul_tile_kernel<Tout, BI, BJ, WI, WJ, DMA>;
    constexpr size_t lds = 2 * (BI + BJ) * kStep;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)(ti * tj)), WI * WJ * 64, lds, s>>>(L, (int)ti, (int)tj);
    return hipGetLastError();
}

// The tile: the one whose launch keeps the GPU's 256 units busy with the least time
// lost to part-filled rounds; wider tiles read less of P and Q for an output.
struct TileChoice {
    int bi, bj, resident;                // outputs of a tile, workgroups of a unit at once
    double rate;                         // of the 256 x 256 tile's, with all units busy
};
constexpr TileChoice kTiles[] = {{256, 256, 1, 1.0}, {128, 128, 2, 0.8}, {64, 64, 4, 0.4}};

int pick_tile(const Sides& S) {
    int best = 0;
    double least = 0;
    for (int t = 0; t < 3; ++t) {
        const TileChoice& c = kTiles[t];
        const double tiles = (double)ceil_div64(S.I, c.bi) * ceil_div64(S.J, c.bj);
        const double rounds = std::ceil(tiles / (256.0 * c.resident)) * c.resident;
        const double time = rounds * c.bi * c.bj / c.rate;
        if (t == 0 || time < least) best = t, least = time;
    }
    return best;
}

template <typename Tout, bool DMA>
hipError_t run_product(const Layer& L, hipStream_t s) {
    switch (pick_tile(sides_of(L))) {
        case 0: return run_tile<Tout, 256, 256, 2, 4, DMA>(L, s);
        case 1: return run_tile<Tout, 128, 128, 2, 2, DMA>(L, s);
        default: return run_tile<Tout, 64, 64, 2, 2, DMA>(L, s);
    }
}

// ------------------------------------------------------------------ few tokens
// At most 16 GT tokens: bound by the weights' bytes, which are read once.  A
// workgroup takes 16 outputs; its waves divide K in turns of kSlab bytes, straight from
// memory to matrix operands (any address), and add their sums through LDS.
constexpr int kSlab = 256;
constexpr int kFewWaves = 8;
constexpr int kFewTokens = 64;

// Where the tokens come from: codes in memory (Code = int8_t), or values that the
// workgroup codes itself into LDS (float, uint16_t), which costs every workgroup a
// reading of all tokens and saves a launch and the codes' way through memory.
struct FewValues {
    const void* x;
    int64_t token_stride, channel_stride;
};
constexpr int kFewValues = 16384;        // values that a workgroup codes at most (their tokens as a power of two)

// Codes and scales of the M <= 16 tokens, in LDS: codes[m * pitch + k], zeros from K to the pitch.
template <typename T>
__device__ void code_few(const FewValues& V, int M, int K, int pitch, int8_t* codes, float* scales, uint32_t* tops) {
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

template <typename Code, typename Tout, int GT, bool MAP>
__global__ __launch_bounds__(kFewWaves * 64) void matmul_few_kernel(Layer L, FewValues V, int R) {
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
    auto fetch = [&](const int8_t* row, int k0, i32x4* to) {
#pragma unroll
        for (int h = 0; h < H; ++h) __builtin_memcpy(&to[h], row + k0 + h * 64 + q16 * 16, 16);
    };
    auto multiply = [](i32x4 u, i32x4 v, i32x4 c) {
        return MAP ? __builtin_amdgcn_mfma_i32_16x16x64_i8(v, u, c, 0, 0, 0)
                   : __builtin_amdgcn_mfma_i32_16x16x64_i8(u, v, c, 0, 0, 0);
    };
    i32x4 a[H], b[GT][H];
    // the first weights are on their way while the tokens are coded
    const int8_t* w = weights(blockIdx.x);
    const int k_first = wave * kSlab, k_whole = K / kSlab * kSlab;
    if (!kCodes && k_first < k_whole) fetch(w, k_first, a);
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
                    fetch(t[g], k0, b[g]);
                } else {
#pragma unroll
                    for (int h = 0; h < H; ++h) b[g][h] = *reinterpret_cast<const i32x4*>(t[g] + k0 + h * 64 + q16 * 16);
                }
            }
        };
        for (int k0 = k_first; k0 < k_whole; k0 += kFewWaves * kSlab) {
            if (kCodes || k0 != k_first || tile != (int)blockIdx.x) fetch(w, k0, a);
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
        if (i < I && j < J) store_outputs<Tout>(L, i, j, J, sum);
    }
}

template <typename Code, typename Tout, int GT>
hipError_t run_few(const Layer& L, const FewValues& V, hipStream_t s) {
    static_assert(GT <= kFewWaves, "a wave adds up one group of tokens");
    int R = 16;
    while (R > 2 && ceil_div64(L.N, R) < 256) R /= 2;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div64(L.N, R), sizeof(Code) == 1 ? 4096 : 256));
    const size_t lds = sizeof(Code) == 1 ? 0 : (size_t)L.M * few_pitch(L.K);
    if (L.map) matmul_few_kernel<Code, Tout, GT, true><<<grid, kFewWaves * 64, lds, s>>>(L, V, R);
    else matmul_few_kernel<Code, Tout, GT, false><<<grid, kFewWaves * 64, lds, s>>>(L, V, R);
    return hipGetLastError();
}

// Whether the few-token kernel codes M tokens of K channels itself.
bool codes_itself(int64_t M, int K) {
    if (M > 16) return false;
    int p = 1;
    while (p < M) p *= 2;
    return (int64_t)p * K <= kFewValues;
}

template <typename Code>
hipError_t launch_linear_few(const Layer& L, const FewValues& V, dss_dtype out_dtype, hipStream_t s) {
    return out_dtype == DSS_BF16 ? run_few<Code, uint16_t, 1>(L, V, s) : run_few<Code, float, 1>(L, V, s);
}

template <typename Tout>
hipError_t run_few_codes(const Layer& L, hipStream_t s) {
    if (L.M <= 16) return run_few<int8_t, Tout, 1>(L, FewValues{}, s);
    if (L.M <= 32) return run_few<int8_t, Tout, 2>(L, FewValues{}, s);
    return run_few<int8_t, Tout, 4>(L, FewValues{}, s);
}

hipError_t launch_matmul(const Layer& L, dss_dtype out_dtype, hipStream_t s) {
    if (L.M <= kFewTokens) return out_dtype == DSS_BF16 ? run_few_codes<uint16_t>(L, s) : run_few_codes<float>(L, s);
    auto whole = [](const int8_t* p, int64_t stride, int64_t rows) {
        return (uintptr_t)p % 16 == 0 && (stride % 16 == 0 || rows == 1);
    };
    const bool dma = L.K % 16 == 0 && whole(L.codes, L.codes_stride, L.M) && whole(L.weight, L.weight_stride, L.N);
    // a launch has fewer than 2^32 threads
    const int64_t slab = std::max<int64_t>(256, (((int64_t)1 << 34) / L.N) / 256 * 256);
    for (int64_t m = 0; m < L.M; m += slab) {
        Layer S = L;
        S.M = std::min(L.M - m, slab);
        S.codes += m * L.codes_stride;
        S.scales += m;
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        hipError_t e;
        if (out_dtype == DSS_BF16) e = dma ? run_product<uint16_t, true>(S, s) : run_product<uint16_t, false>(S, s);
        else e = dma ? run_product<float, true>(S, s) : run_product<float, false>(S, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxK = 131071;
constexpr int kMaxN = 1 << 20;

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

// The codes' row length in a workspace: whole 16-byte units.
int padded_k(int K) { return (K + 15) / 16 * 16; }

// Checks of what dss_matmul_tokens and dss_linear_tokens share.
dss_status check_layer(int64_t M, const int8_t* weight, int64_t weight_stride, const float* weight_scales, int32_t N,
                       int32_t K, const float* bias, dss_act act, const void* out, dss_dtype out_dtype,
                       int64_t out_token_stride, int64_t out_channel_stride) {
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (act != DSS_ACT_NONE && act != DSS_ACT_RELU && act != DSS_ACT_TANH)
        return fail(DSS_E_INVALID, "unknown activation %d", act);
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (K > kMaxK)
        return fail(DSS_E_UNSUPPORTED, "a sum of %d products of 8-bit codes may leave 32 bits (at most %d)", K, kMaxK);
    if (weight_stride < K) return fail(DSS_E_INVALID, "weight_stride %lld is less than %d", (long long)weight_stride, K);
    const bool rows = (out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1);
    const bool map = (out_token_stride == 1 || M <= 1) && (out_channel_stride >= M || N == 1);
    if (!rows && !map)
        return fail(out_channel_stride == 1 || out_token_stride == 1 ? DSS_E_INVALID : DSS_E_UNSUPPORTED,
                    "output strides %lld (tokens) and %lld (channels)", (long long)out_token_stride,
                    (long long)out_channel_stride);
    if (!weight || !weight_scales || (uintptr_t)weight_scales % 4 != 0 || (uintptr_t)bias % 4 != 0)
        return fail(DSS_E_INVALID, "weight or weight_scales is NULL, or the scales or the bias are not aligned");
    if (M > 0 && (!out || (uintptr_t)out % dtype_size(out_dtype) != 0))
        return fail(DSS_E_INVALID, "out is NULL or not aligned to its elements");
    return DSS_OK;
}

int64_t workspace_bytes_of(int64_t M, int32_t N, int32_t K, bool from_codes) {
    (void)N;
    return from_codes || codes_itself(M, K) ? 0 : align256(M * 4) + align256(M * padded_k(K));
}

dss_status check_room(int64_t need, const void* workspace, int64_t workspace_bytes) {
    if (need == 0) return DSS_OK;
    if (!workspace || ((uintptr_t)workspace & 255u) != 0)
        return fail(DSS_E_INVALID, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(DSS_E_SHAPE, "workspace of %lld bytes is smaller than the %lld bytes needed",
                    (long long)workspace_bytes, (long long)need);
    return DSS_OK;
}

// The output's orientation: as rows where both would do.
bool is_map(int64_t M, int32_t N, int64_t out_token_stride, int64_t out_channel_stride) {
    return !((out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1));
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_tokens_workspace(int64_t M, int32_t N, int32_t K, int32_t from_codes,
                                           int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    *workspace_bytes = workspace_bytes_of(M, N, K, from_codes != 0);
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_matmul_tokens(const int8_t* codes, int64_t codes_stride, const float* scales, int64_t M,
                                        const int8_t* weight, int64_t weight_stride, const float* weight_scales,
                                        int32_t N, int32_t K, const float* bias, dss_act act, void* out,
                                        dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                        void* workspace, int64_t workspace_bytes, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_layer(M, weight, weight_stride, weight_scales, N, K, bias, act, out, out_dtype,
                               out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    if (codes_stride < K) return fail(DSS_E_INVALID, "codes_stride %lld is less than %d", (long long)codes_stride, K);
    if (M == 0) return DSS_OK;
    if (!codes || !scales || (uintptr_t)scales % 4 != 0)
        return fail(DSS_E_INVALID, "codes or scales is NULL or not aligned to its elements");
    s = check_room(workspace_bytes_of(M, N, K, true), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const Layer L = {codes, codes_stride, scales, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out,
                     map ? out_channel_stride : out_token_stride, map};
    hipError_t e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_linear_tokens(const void* x, dss_dtype dtype, int64_t M, int64_t token_stride,
                                        int64_t channel_stride, const int8_t* weight, int64_t weight_stride,
                                        const float* weight_scales, int32_t N, int32_t K, const float* bias,
                                        dss_act act, void* out, dss_dtype out_dtype, int64_t out_token_stride,
                                        int64_t out_channel_stride, void* workspace, int64_t workspace_bytes,
                                        hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    s = check_layer(M, weight, weight_stride, weight_scales, N, K, bias, act, out, out_dtype, out_token_stride,
                    out_channel_stride);
    if (s != DSS_OK) return s;
    if (M == 0) return DSS_OK;
    s = check_room(workspace_bytes_of(M, N, K, false), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const int64_t ldo = map ? out_channel_stride : out_token_stride;
    if (codes_itself(M, K)) {
        const Layer L = {nullptr, 0, nullptr, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out, ldo, map};
        const FewValues V = {x, token_stride, channel_stride};
        hipError_t e = dtype == DSS_BF16 ? launch_linear_few<uint16_t>(L, V, out_dtype, stream)
                                         : launch_linear_few<float>(L, V, out_dtype, stream);
        return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
    }
    float* scales = static_cast<float*>(workspace);
    int8_t* codes = static_cast<int8_t*>(workspace) + align256(M * 4);
    const int Kp = padded_k(K);
    hipError_t e = launch_quantize_tokens(dtype, x, M, K, token_stride, channel_stride, codes, Kp, Kp, scales, stream);
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    const Layer L = {codes, Kp, scales, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out, ldo, map};
    e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}
