// Products in microscaled 4-bit floating point where one side has few rows: a server's single tokens
// with a layer's weights, or many tokens with the weights of few outputs.
//
// Bound by the bytes of the other side, which are read once, straight from memory to matrix operands.
// A wave takes R of its rows and a part of K in turns of kSlab blocks; the parts' sums are added
// through LDS in the order of K.
#include <algorithm>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"

namespace dss {

namespace {

constexpr int kSlab = 16;                // blocks: four matrix instructions
constexpr int kWaves = 8;

// The streamed rows s, the few rows f, and D[s][f]: ADJ says whether s is the output's adjacent axis.
struct FewSides {
    Mx4Rows S, F;
    int bias_on_s;
};

template <typename Tout, int GT, bool ADJ>
__global__ __launch_bounds__(kWaves * 64) void matmul_few_mx4_kernel(Mx4Layer L, FewSides D, int R, int parts) {
    __shared__ f32x4 sums[kWaves][GT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, q16 = lane >> 4;
    const int part = wave % parts;
    const int64_t s0 = ((int64_t)blockIdx.x * (kWaves / parts) + wave / parts) * R;
    const int64_t s = min(s0 + min(l16, R - 1), D.S.rows - 1);
    const uint8_t *codes_s = D.S.codes + s * D.S.stride, *scale_s = D.S.scales + s;
    const uint8_t *codes_f[GT], *scale_f[GT];
#pragma unroll
    for (int g = 0; g < GT; ++g) {
        const int64_t f = min((int64_t)(g * 16 + l16), D.F.rows - 1);
        codes_f[g] = D.F.codes + f * D.F.stride;
        scale_f[g] = D.F.scales + f;
    }
    f32x4 acc[GT] = {};
    for (int64_t b0 = (int64_t)part * kSlab; b0 < L.B; b0 += (int64_t)parts * kSlab) {
        i32x4 a[kSlab / 4];
        uint32_t x[kSlab / 4];
#pragma unroll
        for (int h = 0; h < kSlab / 4; ++h) {
            // past the end of K: the last block with zeros for one side's codes (its scales count already)
            const int64_t b = min(b0 + h * 4 + q16, (int64_t)L.B - 1);
            a[h] = *reinterpret_cast<const i32x4*>(codes_s + b * 16);
            if (b != b0 + h * 4 + q16) a[h] = i32x4{};
            x[h] = scale_s[b * D.S.scales_stride];
        }
#pragma unroll
        for (int h = 0; h < kSlab / 4; ++h) {
            const int64_t b = min(b0 + h * 4 + q16, (int64_t)L.B - 1);
#pragma unroll
            for (int g = 0; g < GT; ++g) {
                const i32x4 v = *reinterpret_cast<const i32x4*>(codes_f[g] + b * 16);
                const uint32_t y = scale_f[g][b * D.F.scales_stride];
                acc[g] = ADJ ? multiply_byte<0>(a[h], x[h], v, y, acc[g]) : multiply_byte<0>(v, y, a[h], x[h], acc[g]);
            }
        }
    }
#pragma unroll
    for (int g = 0; g < GT; ++g) sums[wave][g][lane] = acc[g];
    __syncthreads();
    for (int g = part; g < GT; g += parts) {
        f32x4 sum = sums[wave - part][g][lane];
        for (int p = 1; p < parts; ++p) sum += sums[wave - part + p][g][lane];
        const int64_t s_end = min(s0 + R, D.S.rows);
        const int64_t i = ADJ ? g * 16 + l16 : s0 + l16, j = ADJ ? s0 + q16 * 4 : g * 16 + q16 * 4;
        const int64_t I = ADJ ? D.F.rows : s_end, J = ADJ ? s_end : D.F.rows;
        if (i >= I || j >= J) continue;
        const bool bias_on_j = ADJ == (D.bias_on_s != 0);
        float v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            v[k] = activate_nan(L.act, sum[k] + (L.bias ? L.bias[bias_on_j ? min(j + k, J - 1) : i] : 0.f));
        store_values(static_cast<Tout*>(L.out) + i * L.ldo + j, v, j, J, 0);
    }
}

template <typename Tout, int GT>
hipError_t run_few(const Mx4Layer& L, const FewSides& D, bool adj, hipStream_t s) {
    // as many waves share K as have a slab of it; few rows are spread over all units
    int parts = 1, R = 16;
    while (parts < kWaves && parts * kSlab < L.B) parts *= 2;
    while (R > 2 && ceil_div64(D.S.rows, R * (kWaves / parts)) < 256) R /= 2;
    const int64_t groups = ceil_div64(D.S.rows, R * (kWaves / parts));
    const auto kern = adj ? matmul_few_mx4_kernel<Tout, GT, true> : matmul_few_mx4_kernel<Tout, GT, false>;
    // a launch has fewer than 2^32 threads
    const int64_t most = (int64_t)1 << 22, rows = most * R * (kWaves / parts);
    for (int64_t at = 0; at < groups; at += most) {
        Mx4Layer P = L;
        FewSides E = D;
        const int64_t s0 = at / most * rows;
        E.S.codes += s0 * D.S.stride;
        E.S.scales += s0;
        E.S.rows = std::min(rows, D.S.rows - s0);
        P.out = static_cast<Tout*>(L.out) + s0 * (adj ? 1 : L.ldo);
        if (L.bias && D.bias_on_s) P.bias += s0;
        kern<<<dim3((unsigned)std::min(most, groups - at)), kWaves * 64, 0, s>>>(P, E, R, parts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_few_mx4(const Mx4Layer& L, dss_dtype out_dtype, hipStream_t s) {
    const bool tokens = L.tokens.rows <= kFewRows;       // else the outputs are few
    const FewSides D = tokens ? FewSides{L.weight, L.tokens, 1} : FewSides{L.tokens, L.weight, 0};
    const bool adj = tokens != (L.map != 0);
    if (D.F.rows > 16) return out_dtype == DSS_BF16 ? run_few<uint16_t, 2>(L, D, adj, s) : run_few<float, 2>(L, D, adj, s);
    return out_dtype == DSS_BF16 ? run_few<uint16_t, 1>(L, D, adj, s) : run_few<float, 1>(L, D, adj, s);
}

}  // namespace dss
