// Fully connected layers in microscaled 4-bit floating point:
//   y[m][n] = act(sum_b X[b][m] W[b][n] sum_{k in b} q[m][k] v[n][k] + bias[n]),
// on v_mfma_scale_f32_16x16x128_f8f6f4, whose binary32 sums take the blocks' scales with them.
//
// Bound by the matrix units where all sides are large: 8192 x 8192 x 8192 to bfloat16 297 to 303 us in long runs of calls, 3.65
// PFLOP/s (a library's product of the same format 340 us), and 320 to 350 in the first hundred after a pause; by latency where
// they are not: 1777 x 2305 x 1003 11 to 14 us.
#include <algorithm>
#include <type_traits>

#include "dev_common.h"
#include "dss_internal.h"
#include "mx4.h"
#include "mx4_device.h"
#include "tile_choice.h"

namespace dss {

namespace {

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

// ------------------------------------------------------------------ tiles
// D[i][j] = sum_k P[i][k] Q[j][k] with the output's adjacent axis as j: for rows P are the tokens and Q the
// weights, for dense maps the other way round.  In the matrix instruction Q's rows are the result's
// rows, so that a lane holds four adjacent outputs.
//
// BI x BJ outputs for WI x WJ waves; kStep bytes of K (256 channels) at a time through two LDS buffers.
//
// A matrix operand is 16 rows.  Of P they are TI apart: row l of operand a is l TI + a, so that a lane's
// scales for its TI operands are adjacent bytes and come with one load.  Of Q they are adjacent for binary32 outputs, where a
// lane's four outputs are a store of 16 bytes and four lanes write 64 adjacent bytes; for
// bfloat16 outputs two operands share 32 rows, so that a lane has eight adjacent outputs over
// both and the same holds; its scales come byte by byte.  A row of a buffer is 8 units of 16 bytes, a block's codes each; a
// row that is an operand's row l keeps unit u at place u ^ (l & 7): the 8 rows that the operand's
// read takes at once lie in different banks.
constexpr int kUnits = kStep / 16;

// 16 zero bytes: the source of the blocks past the end of K.
__device__ __attribute__((aligned(16))) const unsigned int g_zero16[4] = {0u, 0u, 0u, 0u};

typedef __attribute__((address_space(3))) void lds_void;

// 16 bytes of each lane from global memory to LDS at wave_dst + 16 * lane.
__device__ __forceinline__ void copy16(const void* src, char* wave_dst) {
    __builtin_amdgcn_global_load_lds(src, (lds_void*)wave_dst, 16, 0, 0);
}

// N adjacent scales, in the low bytes.
template <int N>
struct Scales {
    uint32_t w[(N + 3) / 4];
};
template <int N>
__device__ __forceinline__ Scales<N> load_scales(const uint8_t* p, int shift) {
    Scales<N> r = {};
    if constexpr (N == 8) {
        uint64_t v;
        __builtin_memcpy(&v, p, 8);
        v >>= shift;
        r.w[0] = (uint32_t)v;
        r.w[1] = (uint32_t)(v >> 32);
    } else {
        __builtin_memcpy(r.w, p, N);
        r.w[0] >>= shift;
    }
    return r;
}

struct Sides {
    Mx4Rows P, Q;
};
__host__ __device__ __forceinline__ Sides sides_of(const Mx4Layer& L) {
    if (L.map) return {L.weight, L.tokens};
    return {L.tokens, L.weight};
}

// A lane's outputs of a tile: of rows i .. i+TI-1, C adjacent ones from j on, and every 4 C further.
template <typename Tout, int TI, int TJ, bool MAP>
__device__ __forceinline__ void store_tile(const Mx4Layer& L, const f32x4 (&acc)[TI][TJ], int64_t i_lane, int64_t I, int64_t j, int64_t J) {
    constexpr int C = 16 / (int)sizeof(Tout);
    constexpr int STORES = TJ * 4 / C;
    float bias_j[STORES][C] = {};
    if (!MAP && L.bias) {
#pragma unroll
        for (int c = 0; c < STORES; ++c)
#pragma unroll
            for (int k = 0; k < C; ++k) bias_j[c][k] = L.bias[min(j + c * 4 * C + k, J - 1)];
    }
    float bias_i[TI] = {};
    if (MAP && L.bias) {
#pragma unroll
        for (int a = 0; a < TI; ++a) bias_i[a] = L.bias[min(i_lane + a, I - 1)];
    }
#pragma unroll
    for (int a = 0; a < TI; ++a) {
        const int64_t i = i_lane + a;
#pragma unroll
        for (int c = 0; c < STORES; ++c) {
            if (i >= I || j + c * 4 * C >= J) continue;
            float v[C];
#pragma unroll
            for (int k = 0; k < C; ++k)
                v[k] = acc[a][c * (C / 4) + k / 4][k % 4] + (MAP ? bias_i[a] : bias_j[c][k]);
            activate_all(L.act, v);
            store_values(static_cast<Tout*>(L.out) + i * L.ldo + j + c * 4 * C, v, j + c * 4 * C, J, L.past);
        }
    }
}

template <typename Tout, int BI, int BJ, int WI, int WJ, bool MAP>
__global__ __launch_bounds__(WI* WJ * 64) __attribute__((amdgpu_waves_per_eu(2)))
void matmul_mx4_kernel(Mx4Layer L, int tiles_i, int tiles_j) {
    constexpr int NW = WI * WJ, THREADS = NW * 64;
    constexpr int TI = BI / WI / 16, TJ = BJ / WJ / 16;
    constexpr int C = 16 / (int)sizeof(Tout);            // outputs of a store, from C / 4 operands of Q
    constexpr int LP = BI * kUnits / THREADS, LQ = BJ * kUnits / THREADS;   // units of each thread and step
    static_assert(LP * THREADS == BI * kUnits && LQ * THREADS == BJ * kUnits && THREADS % 64 == 0, "tile");
    static_assert(TI <= 8 && THREADS / 8 % (8 * TI) == 0 && THREADS / 8 % 32 == 0 && TJ % (C / 4) == 0,
                  "the places of a thread's units, the operands of a store");
    constexpr int BUF = (BI + BJ) * kStep;
    extern __shared__ __align__(16) char lds[];
    const Sides S = sides_of(L);
    const int64_t I = S.P.rows, J = S.Q.rows;
    // tiles in strips of 8 along i: a strip's tiles share their rows of Q in cache
    const int64_t id = xcd_order(blockIdx.x, (int64_t)tiles_i * tiles_j);
    const int64_t strip = id / ((int64_t)8 * tiles_j), in_strip = id - strip * 8 * tiles_j;
    const int rows = min(8, tiles_i - (int)strip * 8);
    const int64_t i0 = (strip * 8 + in_strip % rows) * BI, j0 = in_strip / rows * BJ;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q16 = lane >> 4;
    const int wi = wave / WJ, wj = wave % WJ;

    // the thread's units: rows row0 + n * (THREADS / 8), and one place in each of them.  Their
    // offsets from the tile's first rows fit 32 bits (kMostStride).
    const int row0 = tid >> 3;
    const int unit_p = (tid & 7) ^ (row0 / TI & 7), unit_q = (tid & 7) ^ ((row0 & 3) | (row0 / C & 1) << 2);
    const uint8_t *const base_p = S.P.codes + i0 * S.P.stride, *const base_q = S.Q.codes + j0 * S.Q.stride;
    uint32_t src_p[LP], src_q[LQ];
#pragma unroll
    for (int n = 0; n < LP; ++n) src_p[n] = (uint32_t)min((int64_t)row0 + n * (THREADS / 8), I - 1 - i0) * (uint32_t)S.P.stride;
#pragma unroll
    for (int n = 0; n < LQ; ++n) src_q[n] = (uint32_t)min((int64_t)row0 + n * (THREADS / 8), J - 1 - j0) * (uint32_t)S.Q.stride;

    const int B = L.B, steps = (B + kUnits - 1) / kUnits;
    f32x4 acc[TI][TJ] = {};

    // Unit n of the thread's LP + LQ units of step s, into the step's buffer; past the end of K zeros.
    const uint8_t* zeros = reinterpret_cast<const uint8_t*>(g_zero16);
    auto fetch = [&](int s, int n) {
        const int b = s * kUnits + (n < LP ? unit_p : unit_q);
        const uint8_t* row = n < LP ? base_p + src_p[n < LP ? n : 0] : base_q + src_q[n < LP ? 0 : n - LP];
        copy16(b < B ? row + (int64_t)b * 16 : zeros, lds + (s & 1) * BUF + (n * NW + wave) * 1024);
    };
    // A barrier that waits for the wave's own copies first: they count as loads, for which a barrier
    // alone does not wait.
    auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // The scales of half a step (4 blocks): the lane's block is b.  Past the end of K, where the codes are zeros, the
    // last block's (if that is NaN, so are the outputs already).  The last rows' loads end with them.
    const int64_t i_lane = i0 + wi * TI * 16 + l16 * TI, i_at = min(i_lane, I - TI);
    const int shift_p = 8 * (int)min(i_lane - i_at, (int64_t)TI - 1);
    uint32_t off_q[TJ];
#pragma unroll
    for (int n = 0; n < TJ; ++n)
        off_q[n] = (uint32_t)min(j0 + wj * TJ * 16 + (l16 >> 2) * C + (l16 & 3) + n / (C / 4) * 4 * C + n % (C / 4) * 4, J - 1);
    struct Half {
        i32x4 o[TI + TJ];
        Scales<TI> p;
        uint32_t q[TJ];
    };
    auto scales = [&](Half& o, int s, int h) {
        const int64_t b = min(s * kUnits + h * 4 + q16, B - 1);
        o.p = load_scales<TI>(S.P.scales + b * S.P.scales_stride + i_at, shift_p);
        const uint8_t* q = S.Q.scales + b * S.Q.scales_stride;
#pragma unroll
        for (int n = 0; n < TJ; ++n) o.q[n] = q[off_q[n]];
    };

    // The matrix operands of half a step: TJ of Q, then TI of P.
    const int at_p = (wi * TI * 16 + l16 * TI) * kStep;
    const int at_q = (BI + wj * TJ * 16 + (l16 >> 2) * C + (l16 & 3)) * kStep;
    auto read = [&](Half& o, int n, int s, int h) {
        const int at = n < TJ ? at_q + (n / (C / 4) * 4 * C + n % (C / 4) * 4) * kStep : at_p + (n - TJ) * kStep;
        o.o[n] = *reinterpret_cast<const i32x4*>(lds + (s & 1) * BUF + at + ((h * 4 + q16) ^ (l16 & 7)) * 16);
    };
    // Multiplies one half's operands, reads another's (half h of step s) and fetches a step's
    // units, an LDS read and a fetch after every few matrix instructions.  In a burst the fetches would
    // hold up the wave, and with it its matrix instructions, until all of them are taken.
    auto half_step = [&](Half& use, Half& next, int s, int h, bool fetches) {
        constexpr int R = TI + TJ;
        scales(next, s, h);
#pragma unroll
        for (int n = 0; n < R; ++n) {
            if (fetches)
#pragma unroll
                for (int f = (LP + LQ) * n / R; f < (LP + LQ) * (n + 1) / R; ++f) fetch(s + 1, f);
            read(next, n, s, h);
#pragma unroll
            for (int m = TI * TJ * n / R; m < TI * TJ * (n + 1) / R; ++m)
                acc[m / TJ][m % TJ] = multiply_at(m / TJ, use.o[m % TJ], use.q[m % TJ], use.o[TJ + m / TJ], use.p.w[m / TJ / 4],
                                                  acc[m / TJ][m % TJ]);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // A step's second half is read while its first is multiplied.  Then nobody needs the step's
    // buffer any more, and the next step's bytes have had a step's time to arrive: one barrier for
    // both, after which the buffer takes the step after the next and the next one's first half is read.
    // (Past the last step zeros are fetched and read, and not used: no branch divides the loop.)
#pragma unroll
    for (int s = 0; s < 2; ++s) {
#pragma unroll
        for (int n = 0; n < LP + LQ; ++n) fetch(s, n);
    }
    Half h0, h1;
    scales(h0, 0, 0);
    arrived();
#pragma unroll
    for (int n = 0; n < TI + TJ; ++n) read(h0, n, 0, 0);
    for (int s = 0; s < steps; ++s) {
        half_step(h0, h1, s, 1, false);
        arrived();
        half_step(h1, h0, s + 1, 0, true);
    }
    arrived();                           // no copy may outlive the workgroup
    store_tile<Tout, TI, TJ, MAP>(L, acc, i_lane, I, j0 + wj * TJ * 16 + q16 * C, J);
}

// ------------------------------------------------------------------ small tiles
// Where a step's matrix instructions take less time than its bytes need to arrive: NB buffers, so that NB - 1 steps are
// on their way, and all scales of the tile's rows in LDS beforehand (a load into registers between the copies would have
// to wait for those before it).  (BI + BJ) B bytes of LDS for them.
template <typename Tout, int BI, int BJ, int NB, bool MAP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2)))
void matmul_mx4_deep_kernel(Mx4Layer L, int tiles_i, int tiles_j) {
    constexpr int WI = 2, WJ = 2, NW = 4, THREADS = 256;
    constexpr int TI = BI / WI / 16, TJ = BJ / WJ / 16;
    constexpr int C = 16 / (int)sizeof(Tout);
    constexpr int LP = BI * kUnits / THREADS, LQ = BJ * kUnits / THREADS;
    constexpr int BUF = (BI + BJ) * kStep;
    static_assert(32 % (8 * TI) == 0 && TJ % (C / 4) == 0, "the places of a thread's units, the operands of a store");
    extern __shared__ __align__(16) char lds[];
    const Sides S = sides_of(L);
    const int64_t I = S.P.rows, J = S.Q.rows;
    const int64_t id = xcd_order(blockIdx.x, (int64_t)tiles_i * tiles_j);
    const int64_t strip = id / ((int64_t)8 * tiles_j), in_strip = id - strip * 8 * tiles_j;
    const int strip_rows = min(8, tiles_i - (int)strip * 8);
    const int64_t i0 = (strip * 8 + in_strip % strip_rows) * BI, j0 = in_strip / strip_rows * BJ;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q16 = lane >> 4, wi = wave / WJ, wj = wave % WJ;
    const int B = L.B, steps = (B + kUnits - 1) / kUnits;
    uint8_t* const scales = reinterpret_cast<uint8_t*>(lds) + NB * BUF;      // [B][BI + BJ]

    // Four adjacent rows' scales of a block at a time, U of them under way; past a side's end any.
    constexpr int U = 8, FOURS = (BI + BJ) / 4;
    auto load_four = [&](int n) {
        const int b = min(n / FOURS, B - 1), r = n % FOURS * 4;
        const bool p = r < BI;
        const int64_t at = p ? i0 + r : j0 + r - BI, rows = p ? I : J;
        const uint8_t* from = p ? S.P.scales + b * S.P.scales_stride : S.Q.scales + b * S.Q.scales_stride;
        const int64_t start = min(at, rows - 4);         // (the rows before `at` are shifted out)
        uint32_t w;
        __builtin_memcpy(&w, from + start, 4);
        return w >> 8 * (int)min(at - start, (int64_t)3);
    };
    auto put_fours = [&](int n0, const uint32_t (&w)[U]) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (n0 + u * THREADS < B * FOURS) reinterpret_cast<uint32_t*>(scales)[n0 + u * THREADS] = w[u];
    };
    uint32_t fours[U];
#pragma unroll
    for (int u = 0; u < U; ++u) fours[u] = load_four(tid + u * THREADS);

    const int row0 = tid >> 3;
    const int unit_p = (tid & 7) ^ (row0 / TI & 7), unit_q = (tid & 7) ^ ((row0 & 3) | (row0 / C & 1) << 2);
    const uint8_t *const base_p = S.P.codes + i0 * S.P.stride, *const base_q = S.Q.codes + j0 * S.Q.stride;
    uint32_t src_p[LP], src_q[LQ];
#pragma unroll
    for (int n = 0; n < LP; ++n) src_p[n] = (uint32_t)min((int64_t)row0 + n * 32, I - 1 - i0) * (uint32_t)S.P.stride;
#pragma unroll
    for (int n = 0; n < LQ; ++n) src_q[n] = (uint32_t)min((int64_t)row0 + n * 32, J - 1 - j0) * (uint32_t)S.Q.stride;
    const uint8_t* zeros = reinterpret_cast<const uint8_t*>(g_zero16);
    auto fetch = [&](int s, char* buffer) {
#pragma unroll
        for (int n = 0; n < LP + LQ; ++n) {
            const int b = s * kUnits + (n < LP ? unit_p : unit_q);
            const uint8_t* row = n < LP ? base_p + src_p[n < LP ? n : 0] : base_q + src_q[n < LP ? 0 : n - LP];
            copy16(b < B ? row + (int64_t)b * 16 : zeros, buffer + (n * NW + wave) * 1024);
        }
    };
    const int at_p = (wi * TI * 16 + l16 * TI) * kStep;
    const int at_q = (BI + wj * TJ * 16 + (l16 >> 2) * C + (l16 & 3)) * kStep;
    const uint8_t* const scales_p = scales + wi * TI * 16 + l16 * TI;
    const uint8_t* const scales_q = scales + BI + wj * TJ * 16 + (l16 >> 2) * C;
    const int shift_q = 8 * (l16 & 3);
    // (words, not bytes: a byte might be one that a copy writes, and its read would wait for all of them)
    using Word = std::conditional_t<TI == 2, uint16_t, uint32_t>;
    static_assert(TI == (int)sizeof(Word));

    f32x4 acc[TI][TJ] = {};
    char* next = lds;                    // the buffer that the next fetch takes
    auto turn = [&](char* b) { return b + BUF == lds + NB * BUF ? lds : b + BUF; };
#pragma unroll
    for (int s = 0; s < NB - 1; ++s) {
        fetch(s, next);
        next = turn(next);
    }
    put_fours(tid, fours);
    for (int n0 = tid + U * THREADS; n0 < B * FOURS; n0 += U * THREADS) {
#pragma unroll
        for (int u = 0; u < U; ++u) fours[u] = load_four(n0 + u * THREADS);
        put_fours(n0, fours);
    }
    char* use = lds;
    for (int s = 0; s < steps; ++s) {
        // step s has arrived, for all waves, and nobody reads the buffer of step s - 1 any more
        // (a barrier of the language would wait for all copies)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"((NB - 2) * (LP + LQ)) : "memory");
        fetch(s + NB - 1, next);         // (past the last step zeros, which are not used)
        next = turn(next);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            i32x4 p[TI], q[TJ];
            const int unit = ((h * 4 + q16) ^ (l16 & 7)) * 16, b = min(s * kUnits + h * 4 + q16, B - 1);
#pragma unroll
            for (int n = 0; n < TJ; ++n)
                q[n] = *reinterpret_cast<const i32x4*>(use + at_q + (n / (C / 4) * 4 * C + n % (C / 4) * 4) * kStep + unit);
#pragma unroll
            for (int n = 0; n < TI; ++n) p[n] = *reinterpret_cast<const i32x4*>(use + at_p + n * kStep + unit);
            const uint32_t x = *reinterpret_cast<const Word*>(scales_p + b * (BI + BJ));
#pragma unroll
            for (int n = 0; n < TJ; ++n) {
                const uint8_t* from = scales_q + b * (BI + BJ) + n / (C / 4) * 4 * C + n % (C / 4) * 4;
                const uint32_t y = *reinterpret_cast<const uint32_t*>(from) >> shift_q;
#pragma unroll
                for (int a = 0; a < TI; ++a) acc[a][n] = multiply_at(a, q[n], y, p[a], x, acc[a][n]);
            }
        }
        use = turn(use);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");     // no copy may outlive the workgroup
    store_tile<Tout, TI, TJ, MAP>(L, acc, i0 + wi * TI * 16 + l16 * TI, I, j0 + wj * TJ * 16 + q16 * C, J);
}

template <typename Tout, int BI, int BJ, int WI, int WJ>
hipError_t run_tile(const Mx4Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int64_t ti = ceil_div64(S.P.rows, BI), tj = ceil_div64(S.Q.rows, BJ);
    const auto kern = L.map ? matmul_mx4_kernel<Tout, BI, BJ, WI, WJ, true>
                            : matmul_mx4_kernel<Tout, BI, BJ, WI, WJ, false>;
    constexpr size_t lds = 2 * (BI + BJ) * kStep;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)(ti * tj)), WI * WJ * 64, lds, s>>>(L, (int)ti, (int)tj);
    return hipGetLastError();
}

size_t deep_lds(int BI, int BJ, int NB, int B) { return (size_t)(BI + BJ) * (NB * kStep + B); }

template <typename Tout, int BI, int BJ, int NB>
hipError_t run_deep(const Mx4Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int64_t ti = ceil_div64(S.P.rows, BI), tj = ceil_div64(S.Q.rows, BJ);
    const auto kern = L.map ? matmul_mx4_deep_kernel<Tout, BI, BJ, NB, true> : matmul_mx4_deep_kernel<Tout, BI, BJ, NB, false>;
    const size_t lds = deep_lds(BI, BJ, NB, L.B);
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)(ti * tj)), 256, lds, s>>>(L, (int)ti, (int)tj);
    return hipGetLastError();
}

template <typename Tout>
hipError_t run_product(const Mx4Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int t = pick_mx4_tile(S.P.rows, S.Q.rows, L.B);
    if (t == 0) return run_tile<Tout, 256, 256, 2, 4>(L, s);
    if (t == 1) return run_tile<Tout, 128, 128, 2, 2>(L, s);
    return run_deep<Tout, 64, 64, 3>(L, s);
}

// The largest row stride of a tile's operands: 256 rows of them stay in 32 bits.
constexpr int64_t kMostStride = (int64_t)1 << 23;

// The layer on codes.
hipError_t launch_matmul(const Mx4Layer& L, dss_dtype out_dtype, hipStream_t s) {
    const bool few = L.tokens.rows <= kFewRows || L.weight.rows <= kFewRows;
    if (few) return launch_few_mx4(L, out_dtype, s);
    // rows too long for the tiles are taken kFewRows at a time; a launch of tiles has fewer than 2^32
    // threads: at most 2^21 tiles of 64 x 64
    const bool tiles = std::max(L.tokens.stride, L.weight.stride) <= kMostStride;
    const int64_t slab = tiles ? std::max<int64_t>(256, (((int64_t)1 << 27) / ceil_div64(L.weight.rows, 64)) / 256 * 256) : kFewRows;
    for (int64_t m = 0; m < L.tokens.rows; m += slab) {
        Mx4Layer S = L;
        S.tokens.rows = std::min(slab, L.tokens.rows - m);
        S.tokens.codes += m * L.tokens.stride;
        S.tokens.scales += m;
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        const bool tile = tiles && S.tokens.rows > kFewRows;
        const hipError_t e = !tile ? launch_few_mx4(S, out_dtype, s)
                             : out_dtype == DSS_BF16 ? run_product<uint16_t>(S, s) : run_product<float>(S, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxN = 1 << 20;
constexpr int kMaxBlocks = 1 << 26;

// Checks of what dss_matmul_blocks and dss_linear_blocks share.
dss_status check_layer(int64_t M, const Mx4Rows& W, int64_t B, const float* bias, dss_act act, const void* out,
                       dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride) {
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (act != DSS_ACT_NONE && act != DSS_ACT_RELU && act != DSS_ACT_TANH)
        return fail(DSS_E_INVALID, "unknown activation %d", act);
    if (M < 0 || M > kMaxTokens || W.rows < 1 || W.rows > kMaxN || B < 1 || B > kMaxBlocks)
        return fail(DSS_E_INVALID, "%lld tokens of %lld blocks, %lld outputs", (long long)M, (long long)B, (long long)W.rows);
    dss_status s = check_mx4_rows(W, B, "weight");
    if (s != DSS_OK) return s;
    if ((uintptr_t)bias % 4 != 0) return fail(DSS_E_INVALID, "bias is not aligned to its elements");
    return check_outputs(M, (int32_t)W.rows, out, out_dtype, out_token_stride, out_channel_stride);
}

// The tokens' codes and scales.
int64_t workspace_bytes_of(int64_t M, int64_t B) { return align256(M * B * 16) + align256(M * B); }

Mx4Layer layer_of(const Mx4Rows& tokens, const Mx4Rows& weight, int64_t B, const float* bias, dss_act act, void* out,
                  dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride) {
    const bool map = is_map(tokens.rows, (int32_t)weight.rows, out_token_stride, out_channel_stride);
    const int64_t ldo = map ? out_channel_stride : out_token_stride;
    return {tokens, weight, (int)B, bias, (int)act, out, ldo, map, outputs_past(tokens.rows, weight.rows, ldo, out, out_dtype)};
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_blocks_workspace(int64_t M, int32_t N, int32_t K, dss_token_source source,
                                        int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (source != DSS_TOKENS_ROWS && source != DSS_TOKENS_MAP && source != DSS_TOKENS_CODES)
        return fail(DSS_E_INVALID, "unknown token source %d", (int)source);
    if (source != DSS_TOKENS_CODES && M > ((int64_t)1 << 62) / (blocks_of(K) * 17))
        return fail(DSS_E_INVALID, "the codes of %lld tokens of %d channels", (long long)M, K);
    const bool none = source == DSS_TOKENS_CODES || few_codes_itself(M, K) || linear_mx4_at_once(M, N, K, source == DSS_TOKENS_MAP);
    *workspace_bytes = none ? 0 : workspace_bytes_of(M, blocks_of(K));
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_matmul_blocks(const uint8_t* codes, int64_t codes_stride, const uint8_t* scales, int64_t scales_stride,
                                     int64_t M, const uint8_t* weight, int64_t weight_stride, const uint8_t* weight_scales,
                                     int64_t weight_scales_stride, int32_t N, int32_t blocks, const float* bias, dss_act act,
                                     void* out, dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                     hipStream_t stream) try {
    using namespace dss;
    const Mx4Rows T = {codes, codes_stride, scales, scales_stride, M};
    const Mx4Rows W = {weight, weight_stride, weight_scales, weight_scales_stride, N};
    dss_status s = check_layer(M, W, blocks, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    s = check_mx4_rows(T, blocks, "tokens");
    if (s != DSS_OK || M == 0) return s;
    const Mx4Layer L = layer_of(T, W, blocks, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    hipError_t e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_linear_blocks(const void* x, dss_dtype dtype, int64_t M, int64_t token_stride, int64_t channel_stride,
                                     const uint8_t* weight, int64_t weight_stride, const uint8_t* weight_scales,
                                     int64_t weight_scales_stride, int32_t N, int32_t K, const float* bias, dss_act act,
                                     void* out, dss_dtype out_dtype, int64_t out_token_stride, int64_t out_channel_stride,
                                     void* workspace, int64_t workspace_bytes, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(x, dtype, M, K, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    const int64_t B = blocks_of(K);
    const Mx4Rows W = {weight, weight_stride, weight_scales, weight_scales_stride, N};
    s = check_layer(M, W, B, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK || M == 0) return s;
    const bool from_map = channel_stride != 1 && K > 1;
    int64_t need = 0;
    s = dss_blocks_workspace(M, N, K, from_map ? DSS_TOKENS_MAP : DSS_TOKENS_ROWS, &need);
    if (s != DSS_OK) return s;
    s = check_room(need, workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool few = few_codes_itself(M, K);
    if (few || linear_mx4_at_once(M, N, K, from_map)) {
        const Mx4Layer L = layer_of({nullptr, 0, nullptr, 0, M}, W, B, bias, act, out, out_dtype, out_token_stride, out_channel_stride);
        const Mx4Values X = {x, dtype, K, token_stride, channel_stride};
        hipError_t e = few ? launch_linear_few_mx4(L, X, out_dtype, stream) : launch_linear_mx4(L, X, out_dtype, stream);
        return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
    }
    uint8_t* codes = static_cast<uint8_t*>(workspace);
    uint8_t* scales = codes + align256(M * B * 16);
    hipError_t e = launch_quantize_mx4(dtype, x, M, K, token_stride, channel_stride, codes, B * 16, scales, M, stream);
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    const Mx4Layer L = layer_of({codes, B * 16, scales, M, M}, W, B, bias, act, out, out_dtype, out_token_stride,
                                out_channel_stride);
    e = launch_matmul(L, out_dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}
