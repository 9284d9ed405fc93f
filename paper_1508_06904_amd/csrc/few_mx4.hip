// Products in microscaled 4-bit floating point where one side has few rows: a server's single tokens
// with a layer's weights, or many tokens with the weights of few outputs.
//
// Bound by the bytes of the other side, which are read once, straight from memory to matrix operands.
// A wave takes R of its rows at a time and a part of K in turns of kSlab blocks, two of them on their way; the parts'
// sums are added through LDS in the order of K.  The few rows' codes are in LDS for all of a workgroup's waves; few tokens
// that are values yet are coded there.
//
// One token of 9216 channels to 512 outputs: 6.4 us in a captured graph, of which an empty launch is 2, and 7.8 between other
// calls; 13 of 4096 to 16384 as codes 12.5 us (36 MB, 2.9 TB/s), as values 16.3 to 17.6, since each workgroup codes them.  Half as many waves for each row (so that all 512 resident
// workgroups have some) took 14.2 and 21.9 us; the few rows loaded 8 at a time, not as they come, 12.5 and 17.5.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

constexpr int kSlab = 16;                // blocks: four matrix instructions
constexpr int kSteps = kSlab / 4;
constexpr int kWaves = 8;

// The streamed rows s, the few rows f, and D[s][f]: ADJ says whether s is the output's adjacent axis.
struct FewSides {
    Mx4Rows S, F;
    int bias_on_s;
};

// The few rows' codes and scales in LDS: 16 bytes more for a row than it has, so that rows start in different banks.
struct Held {
    int B;
    __host__ __device__ int pitch() const { return B * 16 + 16; }
    __host__ __device__ int scale_pitch() const { return (B + 3) / 4 * 4 + 4; }
    __host__ __device__ int64_t bytes(int64_t rows) const { return rows * (pitch() + scale_pitch()); }
};

// Codes what is in memory as values, M <= 16 tokens of K channels, into LDS.
template <typename T>
__device__ __forceinline__ void hold_values(const Mx4Values& X, int M, int B, uint8_t* codes, int pitch, uint8_t* scales, int scale_pitch) {
    const int64_t K = X.channels;
    // (one channel alone has any stride, and its tokens theirs; else those of a map are adjacent)
    if (X.channel_stride == 1 || K == 1) {
        // four lanes for a block, with the loads of U of them under way
        constexpr int U = 4;
        const int quarters = M * B * 4, lane4 = threadIdx.x & 3;
        for (int n0 = threadIdx.x; n0 < (quarters + 63) / 64 * 64; n0 += U * kWaves * 64) {
            Eight<T> v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int n = (n0 + u * kWaves * 64) / 4, m = n / B, b = n - m * B;
                const int64_t k = b * kBlock + lane4 * 8;
                if (n < M * B) v[u].load(static_cast<const T*>(X.x) + m * X.token_stride + k, K - k);
                else v[u].clear();
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int n = (n0 + u * kWaves * 64) / 4, m = n / B, b = n - m * B;
                const uint32_t byte = v[u].scale_byte_of_four();
                if (n >= M * B) continue;
                *reinterpret_cast<uint32_t*>(codes + m * pitch + b * 16 + lane4 * 4) = v[u].codes(byte);
                if (lane4 == 0) scales[m * scale_pitch + b] = (uint8_t)byte;
            }
        }
    } else {
        for (int n = threadIdx.x; n < M * B; n += kWaves * 64) {
            const int b = n / M, m = n - b * M;
            uint32_t byte;
            const i32x4 w = block_codes(static_cast<const T*>(X.x) + m + b * kBlock * X.channel_stride, X.channel_stride,
                                        (int)min((int64_t)kBlock, K - b * kBlock), byte);
            *reinterpret_cast<i32x4*>(codes + m * pitch + b * 16) = w;
            scales[m * scale_pitch + b] = (uint8_t)byte;
        }
    }
}

constexpr int kSums = kWaves * 64 * 16;  // bytes of the parts' sums

// A lane's outputs of rows s0 .. s_end-1: ADJ: four adjacent ones of few row l16; else of row s0 + l16.
template <typename Tout, bool ADJ>
__device__ __forceinline__ void store_few(const Mx4Layer& L, const FewSides& D, f32x4 sum, int64_t s0, int64_t s_end) {
    const int lane = threadIdx.x & 63, l16 = lane & 15, q16 = lane >> 4;
    const int64_t i = ADJ ? l16 : s0 + l16, j = ADJ ? s0 + q16 * 4 : q16 * 4;
    const int64_t I = ADJ ? D.F.rows : s_end, J = ADJ ? s_end : D.F.rows;
    if (i >= I || j >= J) return;
    const bool bias_on_j = ADJ == (D.bias_on_s != 0);
    float v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = sum[k] + (L.bias ? L.bias[bias_on_j ? min(j + k, J - 1) : i] : 0.f);
    activate_all(L.act, v);
    store_values(static_cast<Tout*>(L.out) + i * L.ldo + j, v, j, J, 0);
}

// X: uint8_t where the few rows are codes in memory, else their values' type.
template <typename X, typename Tout, bool ADJ>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(2)))
void matmul_few_mx4_kernel(Mx4Layer L, FewSides D, Mx4Values V, int R, int parts) {
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, q16 = lane >> 4;
    const int part = wave % parts, side = wave / parts, sides = kWaves / parts;
    const int B = L.B, rows_f = (int)D.F.rows, own_f = min(l16, rows_f - 1);
    const Held held = {B};
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);                   // [kWaves][64]
    uint8_t* const codes = lds + kSums;
    uint8_t* const scales = codes + rows_f * held.pitch();
    // (neighbours on one XCD: a line of scales belongs to 128 rows)
    const int64_t first = xcd_order(blockIdx.x, gridDim.x), all = (int64_t)gridDim.x * sides;
    const int64_t tiles = (D.S.rows + R - 1) / R, turns = (tiles - first * sides + all - 1) / all;
    const int slabs = (B + kSlab - 1) / kSlab, own = (slabs - part + parts - 1) / parts;     // of them the wave's

    // A slab of a tile's rows: past the end of K the last block with zeros for its codes (its scales count already).
    struct Slab {
        i32x4 a[kSteps];
        uint32_t x[kSteps];
    };
    auto tile_of = [&](int64_t turn) { return first * sides + turn * all + side; };
    auto fetch = [&](Slab& to, int64_t turn, int n) {
        const int64_t s = min(min(tile_of(turn), tiles - 1) * R + min(l16, R - 1), D.S.rows - 1);
        const uint8_t *c = D.S.codes + s * D.S.stride, *x = D.S.scales + s;
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            const int at = (part + n * parts) * kSlab + h * 4 + q16, b = min(at, B - 1);
            to.a[h] = *reinterpret_cast<const i32x4*>(c + (int64_t)b * 16);
            if (b != at) to.a[h] = i32x4{};
            to.x[h] = x[b * D.S.scales_stride];
        }
    };
    Slab next[2];
    // the first slabs are on their way while the few rows are put into LDS
    int64_t turn1 = 0;                   // the turn and place of the slab to fetch next
    int at1 = 0;
    auto ahead = [&](Slab& to) {
        fetch(to, turn1, at1);
        if (++at1 >= own) at1 = 0, ++turn1;
    };
    if (own > 0) {
        ahead(next[0]);
        ahead(next[1]);
    }
    if constexpr (sizeof(X) == 1) {
        for (int n = threadIdx.x; n < rows_f * B; n += kWaves * 64) {
            const int f = n / B, b = n - f * B;
            *reinterpret_cast<i32x4*>(codes + f * held.pitch() + b * 16) =
                *reinterpret_cast<const i32x4*>(D.F.codes + f * D.F.stride + b * 16);
        }
        for (int n = threadIdx.x; n < rows_f * B; n += kWaves * 64) {
            const int b = n / rows_f, f = n - b * rows_f;
            scales[f * held.scale_pitch() + b] = D.F.scales[b * D.F.scales_stride + f];
        }
    } else {
        hold_values<X>(V, rows_f, B, codes, held.pitch(), scales, held.scale_pitch());
    }
    __syncthreads();
    int buffer = 0;
    for (int64_t turn = 0; turn < turns; ++turn) {
        f32x4 acc = {};
        auto multiply = [&](const Slab& use, int n) {
#pragma unroll
            for (int h = 0; h < kSteps; ++h) {
                const int b = min((part + n * parts) * kSlab + h * 4 + q16, B - 1);
                const i32x4 v = *reinterpret_cast<const i32x4*>(codes + own_f * held.pitch() + b * 16);
                const uint32_t y = scales[own_f * held.scale_pitch() + b];
                acc = ADJ ? multiply_byte<0>(use.a[h], use.x[h], v, y, acc) : multiply_byte<0>(v, y, use.a[h], use.x[h], acc);
            }
        };
        for (int n = 0; n < own; ++n) {
            // (the slabs are named, so that they stay in registers)
            if (buffer == 0) {
                const Slab use = next[0];
                ahead(next[0]);
                multiply(use, n);
            } else {
                const Slab use = next[1];
                ahead(next[1]);
                multiply(use, n);
            }
            buffer ^= 1;
        }
        const int64_t s0 = tile_of(turn) * R;
        if (parts > 1) {
            if (turn) __syncthreads();   // the sums of the last turn have been read
            sums[wave * 64 + lane] = acc;
            __syncthreads();
            if (part > 0) continue;
            for (int p = 1; p < parts; ++p) acc += sums[(wave + p) * 64 + lane];
        }
        store_few<Tout, ADJ>(L, D, acc, s0, min(s0 + R, D.S.rows));
    }
}

// Rows of which LDS does not hold one (over 200 thousand channels): the few rows are read from memory too.
template <typename Tout, bool ADJ>
__global__ __launch_bounds__(kWaves * 64) void matmul_long_mx4_kernel(Mx4Layer L, FewSides D, int R) {
    __shared__ f32x4 sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, q16 = lane >> 4;
    const int64_t s0 = (int64_t)blockIdx.x * R;
    const int64_t s = min(s0 + min(l16, R - 1), D.S.rows - 1);
    const uint8_t *codes_s = D.S.codes + s * D.S.stride, *scale_s = D.S.scales + s;
    const int64_t f = min((int64_t)l16, D.F.rows - 1);
    const uint8_t *codes_f = D.F.codes + f * D.F.stride, *scale_f = D.F.scales + f;
    f32x4 acc = {};
    for (int64_t b0 = (int64_t)wave * kSlab; b0 < L.B; b0 += kWaves * kSlab) {
        i32x4 a[kSteps];
        uint32_t x[kSteps];
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            // past the end of K: the last block with zeros for one side's codes (its scales count already)
            const int64_t b = min(b0 + h * 4 + q16, (int64_t)L.B - 1);
            a[h] = *reinterpret_cast<const i32x4*>(codes_s + b * 16);
            if (b != b0 + h * 4 + q16) a[h] = i32x4{};
            x[h] = scale_s[b * D.S.scales_stride];
        }
#pragma unroll
        for (int h = 0; h < kSteps; ++h) {
            const int64_t b = min(b0 + h * 4 + q16, (int64_t)L.B - 1);
            const i32x4 v = *reinterpret_cast<const i32x4*>(codes_f + b * 16);
            const uint32_t y = scale_f[b * D.F.scales_stride];
            acc = ADJ ? multiply_byte<0>(a[h], x[h], v, y, acc) : multiply_byte<0>(v, y, a[h], x[h], acc);
        }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    for (int p = 1; p < kWaves; ++p) acc += sums[p][lane];
    store_few<Tout, ADJ>(L, D, acc, s0, min(s0 + R, D.S.rows));
}

int64_t lds_of(int B, int64_t rows) { return kSums + Held{B}.bytes(rows); }
constexpr int64_t kMostLds = 160 * 1024;

template <typename X, typename Tout>
hipError_t run_few(const Mx4Layer& L, const FewSides& D, const Mx4Values& V, bool adj, hipStream_t s) {
    // few rows are spread over all units, and K is shared while there are fewer waves than units have room for
    int parts = 1, R = 16;
    while (R > 2 && ceil_div64(D.S.rows, R) < 256) R /= 2;
    while (parts < kWaves && parts * kSlab < L.B && ceil_div64(D.S.rows, R) * parts < 2048) parts *= 2;
    const int64_t groups = ceil_div64(ceil_div64(D.S.rows, R), kWaves / parts);
    const auto kern = adj ? matmul_few_mx4_kernel<X, Tout, true> : matmul_few_mx4_kernel<X, Tout, false>;
    const int64_t lds = lds_of(L.B, D.F.rows);
    const hipError_t e = allow_dynamic_lds((const void*)kern, (size_t)lds);
    if (e != hipSuccess) return e;
    const int64_t resident = 256 * std::max<int64_t>(1, std::min<int64_t>(2, kMostLds / lds));
    kern<<<dim3((unsigned)std::min(groups, resident)), kWaves * 64, (size_t)lds, s>>>(L, D, V, R, parts);
    return hipGetLastError();
}

template <typename Tout>
hipError_t run_long(const Mx4Layer& L, const FewSides& D, bool adj, hipStream_t s) {
    int R = 16;
    while (R > 2 && ceil_div64(D.S.rows, R) < 256) R /= 2;
    const auto kern = adj ? matmul_long_mx4_kernel<Tout, true> : matmul_long_mx4_kernel<Tout, false>;
    // a launch has fewer than 2^32 threads
    const int64_t rows = (int64_t)R << 22;
    for (int64_t at = 0; at < D.S.rows; at += rows) {
        Mx4Layer P = L;
        FewSides E = D;
        E.S.codes += at * D.S.stride;
        E.S.scales += at;
        E.S.rows = std::min(rows, D.S.rows - at);
        P.out = static_cast<Tout*>(L.out) + at * (adj ? 1 : L.ldo);
        if (L.bias && D.bias_on_s) P.bias += at;
        kern<<<dim3((unsigned)ceil_div64(E.S.rows, R)), kWaves * 64, 0, s>>>(P, E, R);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename X>
hipError_t run_types(const Mx4Layer& L, const FewSides& D, const Mx4Values& V, dss_dtype out_dtype, bool adj, hipStream_t s) {
    return out_dtype == DSS_BF16 ? run_few<X, uint16_t>(L, D, V, adj, s) : run_few<X, float>(L, D, V, adj, s);
}

}  // namespace

hipError_t launch_few_mx4(const Mx4Layer& L, dss_dtype out_dtype, hipStream_t s) {
    const bool tokens = L.tokens.rows <= kFewRows;       // else the outputs are few
    const FewSides D = tokens ? FewSides{L.weight, L.tokens, 1} : FewSides{L.tokens, L.weight, 0};
    const bool adj = tokens != (L.map != 0);
    // as many of the few rows at a time as LDS holds
    const int64_t most = (kMostLds - kSums) / Held{L.B}.bytes(1);
    if (most == 0) return out_dtype == DSS_BF16 ? run_long<uint16_t>(L, D, adj, s) : run_long<float>(L, D, adj, s);
    for (int64_t f = 0; f < D.F.rows; f += most) {
        Mx4Layer P = L;
        FewSides E = D;
        E.F.rows = std::min(most, D.F.rows - f);
        E.F.codes += f * D.F.stride;
        E.F.scales += f;
        P.out = static_cast<char*>(L.out) + f * (adj ? L.ldo : 1) * (int64_t)dtype_size(out_dtype);
        if (L.bias && !D.bias_on_s) P.bias += f;
        const hipError_t e = run_types<uint8_t>(P, E, Mx4Values{}, out_dtype, adj, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

// Up to 65536 values: at 16 x 4096 to 4096 outputs the GPU takes 14.4 us for 13.2 in two launches, but the call 10 for 15 where its
// launches are what bounds it; with twice as many values the GPU is what does. Where calls cost nothing, in a captured graph,
// one launch is the faster one for 9216 channels of one token to 512 outputs (6.4 us for 8.9) and the slower one for wide layers
// (13.2 for 11.9 at 16 x 4096 to 4096, 16.3 for 15.7 at 13 x 4096 to 16384), for the workspace that it does without.
bool few_codes_itself(int64_t M, int64_t K) {
    return M <= 16 && M * K <= 65536;
}

hipError_t launch_linear_few_mx4(const Mx4Layer& L, const Mx4Values& X, dss_dtype out_dtype, hipStream_t s) {
    const FewSides D = {L.weight, L.tokens, 1};
    return X.dtype == DSS_BF16 ? run_types<uint16_t>(L, D, X, out_dtype, L.map == 0, s)
                               : run_types<float>(L, D, X, out_dtype, L.map == 0, s);
}

}  // namespace dss
