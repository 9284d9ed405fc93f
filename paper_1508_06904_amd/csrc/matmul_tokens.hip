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
//
// Large products are bound by the matrix units: 8192 x 8192 x 8192 to bfloat16 in 413 to 567 us
// over machines and data (1.9 to 2.7 Pop/s; these units' own rate at the clock they then keep, 1.4
// to 1.8 GHz, would be 2.9 to 3.8), with the matrix pipes busy for two thirds of the time and no
// LDS bank conflict.  Small ones are bound by the steps' latency, those of few channels by their outputs'
// bytes.
#include <algorithm>
#include <cmath>

#include "dev_common.h"
#include "dss_internal.h"
#include "tile_choice.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

// D's operands and extents.
struct Sides {
    const int8_t *P, *Q;
    int64_t ps, qs, I, J;
};
__host__ __device__ __forceinline__ Sides sides_of(const Layer& L) {
    if (L.map) return {L.weight, L.codes, L.weight_stride, L.codes_stride, L.N, L.M};
    return {L.codes, L.weight, L.codes_stride, L.weight_stride, L.M, L.N};
}

// ------------------------------------------------------------------ tiles
// BI x BJ outputs for WI x WJ waves; kStep bytes of K at a time through two LDS
// buffers.  With KG > 1 so many groups of waves take the steps in turn, each with buffers
// of its own: where tiles are fewer than units, a unit has more steps under way.
//
// A matrix operand is 16 rows: of P adjacent ones; of Q adjacent ones too for
// binary32 outputs, where a lane's four outputs are a store of 16 bytes and four lanes
// write 64 adjacent bytes; for bfloat16 outputs two operands share 32 rows, so that a
// lane has eight adjacent outputs over both and the same holds.  A row of a buffer is 8
// units of 16 bytes; a row that is an operand's row l keeps unit u at place u ^ (l & 7):
// the 8 rows that the operand's read takes at once lie in different banks.
//
// The units go from global memory to LDS without a stop in registers; for that rows
// start at 16-byte units, and K ends at one (what does not is copied first).
constexpr int kUnits = kStep / 16;

// 16 zero bytes: the source of the units past the end of K.
__device__ __attribute__((aligned(16))) const unsigned int g_zero16[4] = {0u, 0u, 0u, 0u};

typedef __attribute__((address_space(3))) void lds_void;

// 16 bytes of each lane from global memory to LDS at wave_dst + 16 * lane.
__device__ __forceinline__ void copy16(const void* src, char* wave_dst) {
    __builtin_amdgcn_global_load_lds(src, (lds_void*)wave_dst, 16, 0, 0);
}

template <typename Tout, int BI, int BJ, int WI, int WJ, int KG, bool MAP>
__global__ __launch_bounds__(KG* WI* WJ * 64) __attribute__((amdgpu_waves_per_eu(2))) void matmul_tile_kernel(Layer L, int tiles_i, int tiles_j) {
    constexpr int NW = WI * WJ, THREADS = NW * 64;
    constexpr int TI = BI / WI / 16, TJ = BJ / WJ / 16;
    constexpr int C = 16 / (int)sizeof(Tout);            // outputs of a store, from C / 4 operands of Q
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
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / THREADS), tid = threadIdx.x - group * THREADS;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, q16 = lane >> 4;
    char* const buffers = lds + group * 2 * BUF;
    const int wi = wave / WJ, wj = wave % WJ;

    // the thread's units: rows row0 + n * (THREADS / 8), and one place in each of them
    const int row0 = tid >> 3;
    const int unit_p = (tid & 7) ^ (row0 & 7), unit_q = (tid & 7) ^ ((row0 & 3) | (row0 / C & 1) << 2);
    static_assert(THREADS / 8 % 32 == 0 && TJ % (C / 4) == 0, "the places of a thread's units, the operands of a store");
    const int8_t *src_p[LP], *src_q[LQ];
#pragma unroll
    for (int n = 0; n < LP; ++n) src_p[n] = S.P + min(i0 + row0 + n * (THREADS / 8), S.I - 1) * S.ps;
#pragma unroll
    for (int n = 0; n < LQ; ++n) src_q[n] = S.Q + min(j0 + row0 + n * (THREADS / 8), S.J - 1) * S.qs;

    const int K = L.K, steps = (K + KG * kStep - 1) / (KG * kStep);
    i32x4 acc[TI][TJ] = {};

    // Unit n of the thread's LP + LQ units of step s, into the step's buffer; past the end of K zeros.
    const int8_t* zeros = reinterpret_cast<const int8_t*>(g_zero16);
    auto fetch = [&](int s, int n) {
        const int k = (s * KG + group) * kStep + (n < LP ? unit_p : unit_q) * 16;
        const int8_t* row = n < LP ? src_p[n < LP ? n : 0] : src_q[n < LP ? 0 : n - LP];
        copy16(k < K ? row + k : zeros, buffers + (s & 1) * BUF + (n * NW + wave) * 1024);
    };
    // A barrier that waits for the wave's own copies first: they count as loads, for which a barrier
    // alone does not wait.
    auto arrived = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // The matrix operands of half a step (64 of K): TJ of Q, then TI of P.
    using Half = i32x4[TI + TJ];
    const int at_p = (wi * TI * 16 + l16) * kStep;
    const int at_q = (BI + wj * TJ * 16 + (l16 >> 2) * C + (l16 & 3)) * kStep;
    auto read = [&](Half& o, int n, int s, int h) {
        const int at = n < TJ ? at_q + (n / (C / 4) * 4 * C + n % (C / 4) * 4) * kStep : at_p + (n - TJ) * 16 * kStep;
        o[n] = *reinterpret_cast<const i32x4*>(buffers + (s & 1) * BUF + at + ((h * 4 + q16) ^ (l16 & 7)) * 16);
    };
    // Multiplies one half's operands, reads another's (half h of step s) and fetches a step's
    // units, an LDS read and a fetch after every few matrix instructions.  In a burst the fetches would
    // hold up the wave, and with it its matrix instructions, until all of them are taken.
    auto half_step = [&](Half& use, Half& next, int s, int h, bool fetches) {
        constexpr int R = TI + TJ;
#pragma unroll
        for (int n = 0; n < R; ++n) {
            if (fetches)
#pragma unroll
                for (int f = (LP + LQ) * n / R; f < (LP + LQ) * (n + 1) / R; ++f) fetch(s + 1, f);
            read(next, n, s, h);
#pragma unroll
            for (int m = TI * TJ * n / R; m < TI * TJ * (n + 1) / R; ++m)
                acc[m / TJ][m % TJ] = __builtin_amdgcn_mfma_i32_16x16x64_i8(use[m % TJ], use[TJ + m / TJ], acc[m / TJ][m % TJ], 0, 0, 0);
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
    arrived();
    Half h0, h1;
#pragma unroll
    for (int n = 0; n < TI + TJ; ++n) read(h0, n, 0, 0);
    for (int s = 0; s < steps; ++s) {
        half_step(h0, h1, s, 1, false);
        arrived();
        half_step(h1, h0, s + 1, 0, true);
    }
    arrived();                           // no copy may outlive the workgroup
    if constexpr (KG > 1) {
        // the groups' sums meet in the buffers
        i32x4* sums = reinterpret_cast<i32x4*>(lds) + tid;
#pragma unroll
        for (int n = 0; n < TI * TJ; ++n)
            if (group > 0) sums[((group - 1) * TI * TJ + n) * THREADS] = acc[n / TJ][n % TJ];
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int n = 0; n < TI * TJ; ++n) acc[n / TJ][n % TJ] += sums[(g * TI * TJ + n) * THREADS];
    }
    constexpr int STORES = TJ * 4 / C;
    const int64_t j = j0 + wj * TJ * 16 + q16 * C;
    SideN<C> side_q[STORES];
    Side1 side_p[TI];
#pragma unroll
    for (int c = 0; c < STORES; ++c) side_q[c] = side_j<MAP, C>(L, j + c * 4 * C);
#pragma unroll
    for (int a = 0; a < TI; ++a) side_p[a] = side_i<MAP>(L, i0 + (wi * TI + a) * 16 + l16);
#pragma unroll
    for (int a = 0; a < TI; ++a) {
        const int64_t i = i0 + (wi * TI + a) * 16 + l16;
#pragma unroll
        for (int c = 0; c < STORES; ++c)
            if (i < S.I && j + c * 4 * C < S.J)
                store_outputs<Tout, MAP>(L, i, j + c * 4 * C, S.J, &acc[a][c * (C / 4)], side_p[a], side_q[c]);
    }
}

template <typename Tout, int BI, int BJ, int WI, int WJ, int KG>
hipError_t run_tile(const Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int64_t ti = ceil_div64(S.I, BI), tj = ceil_div64(S.J, BJ);
    const auto kern = L.map ? matmul_tile_kernel<Tout, BI, BJ, WI, WJ, KG, true>
                            : matmul_tile_kernel<Tout, BI, BJ, WI, WJ, KG, false>;
    constexpr size_t lds = KG * 2 * (BI + BJ) * kStep;
    const hipError_t e = allow_dynamic_lds((const void*)kern, lds);
    if (e != hipSuccess) return e;
    kern<<<dim3((unsigned)(ti * tj)), KG * WI * WJ * 64, lds, s>>>(L, (int)ti, (int)tj);
    return hipGetLastError();
}

template <typename Tout>
hipError_t run_product(const Layer& L, hipStream_t s) {
    const Sides S = sides_of(L);
    const int t = pick_tile(S.I, S.J, L.K);
    if (t == 0) return run_tile<Tout, 256, 256, 2, 4, 1>(L, s);
    if (t == 1) return run_tile<Tout, 128, 128, 2, 2, 1>(L, s);
    if (t == 2) return run_tile<Tout, 64, 64, 2, 2, 1>(L, s);
    return run_tile<Tout, 64, 64, 2, 2, 4>(L, s);
}

// ------------------------------------------------------------------ operands at other addresses
// Rows that do not start, or whose K does not end, at 16-byte units, copied with
// zeros up to the next one; a wave for each 4 KB of a row.  Of two operands at once.
struct Rows {
    const int8_t* from;
    int64_t stride, rows;
    int8_t* to;
};

__global__ __launch_bounds__(256) void copy_rows_kernel(Rows A, Rows B, int K, int units) {
    int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    Rows R = A;
    if (row >= A.rows) {
        row -= A.rows;
        R = B;
    }
    if (row >= R.rows) return;
    const int8_t *from = R.from + row * R.stride, *end = R.from + (R.rows - 1) * R.stride + K;
    i32x4* to = reinterpret_cast<i32x4*>(R.to + row * units * 16);
    const int u0 = blockIdx.y * 256 + (threadIdx.x & 63);
    i32x4 v[4];
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if ((u0 + c * 64) * 16 + 16 <= K) v[c] = load_any(from + (u0 + c * 64) * 16, R.from, end);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int u = u0 + c * 64;
        if (u < units) to[u] = u * 16 + 16 <= K ? v[c] : load_unit(from, u * 16, K);
    }
}

bool whole_units(const int8_t* p, int64_t stride, int64_t rows, int K) {
    return K % 16 == 0 && (uintptr_t)p % 16 == 0 && (stride % 16 == 0 || rows == 1);
}

// The codes' row length in a workspace: whole 16-byte units, and of long rows whole lines.
// Units and lines, us for coding and product of 1777 tokens to 2305 outputs: 41/37 from 2305
// channels, 56/50 from 4100, 22.3/21.6 from 1040; 300 to 300 from 2305 18.4/17.0.  (Shorter rows
// gain no less, 24.3/23.1 from 777; only those of 200 are the same.)
int padded_k(int K) { return K >= 1024 ? (K + 127) / 128 * 128 : (K + 15) / 16 * 16; }

int64_t align256(int64_t n) { return (n + 255) / 256 * 256; }

// Tokens whose codes a workspace has room for a copy of: as many as 64 MB hold.
int64_t copied_tokens(int64_t M, int K) {
    return std::min(M, std::max<int64_t>(256, ((int64_t)1 << 26) / padded_k(K) / 256 * 256));
}

// The layer on codes; `room` has the weights' copy and the tokens' (unless these are padded already).
hipError_t launch_matmul(const Layer& L, dss_dtype out_dtype, bool padded, char* room, hipStream_t s) {
    if (few_tokens(L.M, L.N, L.K)) return launch_matmul_few(L, out_dtype, s);
    const int Kp = padded_k(L.K);
    Rows W = {L.weight, L.weight_stride, L.N, reinterpret_cast<int8_t*>(room)};
    int8_t* copies = W.to + align256((int64_t)L.N * Kp);
    const bool copy_w = !whole_units(L.weight, L.weight_stride, L.N, L.K);
    const bool copy_c = !padded && !whole_units(L.codes, L.codes_stride, L.M, L.K);
    // a launch has fewer than 2^32 threads: at most 2^21 tiles of 64 x 64 and 1024 threads
    int64_t slab = std::max<int64_t>(256, (((int64_t)1 << 27) / ceil_div64(L.N, 64)) / 256 * 256);
    if (copy_c) slab = std::min(slab, copied_tokens(L.M, L.K));
    for (int64_t m = 0; m < L.M; m += slab) {
        Layer S = L;
        S.M = std::min(L.M - m, slab);
        S.codes += m * L.codes_stride;
        S.scales += m;
        S.out = static_cast<char*>(L.out) + m * (L.map ? 1 : L.ldo) * (int64_t)dtype_size(out_dtype);
        Rows C = {S.codes, L.codes_stride, copy_c ? S.M : 0, copies};
        Rows w = W;
        if (!copy_w || m > 0) w.rows = 0;
        if (C.rows + w.rows) {
            copy_rows_kernel<<<dim3((unsigned)ceil_div64(C.rows + w.rows, 4), (unsigned)ceil_div64(Kp, 4096)), 256, 0, s>>>(C, w, L.K,
                                                                                                            Kp / 16);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (copy_c) S.codes = copies, S.codes_stride = Kp;
        if (copy_w) S.weight = W.to, S.weight_stride = Kp;
        S.K = (L.K + 15) / 16 * 16;      // (rows that are no copies have no more to read)
        const hipError_t e = out_dtype == DSS_BF16 ? run_product<uint16_t>(S, s) : run_product<float>(S, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

constexpr int kMaxK = 131071;
constexpr int kMaxN = 1 << 20;

dss_status refuse_k(int32_t K) {
    return fail(DSS_E_UNSUPPORTED, "a sum of %d products of 8-bit codes may leave 32 bits (at most %d)", K, kMaxK);
}

// Checks of what dss_matmul_tokens and dss_linear_tokens share.
dss_status check_layer(int64_t M, const int8_t* weight, int64_t weight_stride, const float* weight_scales, int32_t N,
                       int32_t K, const float* bias, dss_act act, const void* out, dss_dtype out_dtype,
                       int64_t out_token_stride, int64_t out_channel_stride) {
    if (out_dtype != DSS_F32 && out_dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d", out_dtype);
    if (act != DSS_ACT_NONE && act != DSS_ACT_RELU && act != DSS_ACT_TANH)
        return fail(DSS_E_INVALID, "unknown activation %d", act);
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (K > kMaxK) return refuse_k(K);
    if (weight_stride < K) return fail(DSS_E_INVALID, "weight_stride %lld is less than %d", (long long)weight_stride, K);
    dss_status s = check_outputs(M, N, out, out_dtype, out_token_stride, out_channel_stride);
    if (s != DSS_OK) return s;
    if (!weight || !weight_scales || (uintptr_t)weight_scales % 4 != 0 || (uintptr_t)bias % 4 != 0)
        return fail(DSS_E_INVALID, "weight or weight_scales is NULL, or the scales or the bias are not aligned");
    return DSS_OK;
}

// The copies of weights and codes (whatever their addresses turn out to be), or the
// weights' copy and the tokens' codes and scales.
int64_t workspace_bytes_of(int64_t M, int32_t N, int32_t K, dss_token_source source) {
    const int64_t Kp = padded_k(K), weights = few_tokens(M, N, K) ? 0 : align256(N * Kp);
    if (source == DSS_TOKENS_CODES) return few_tokens(M, N, K) ? 0 : weights + align256(copied_tokens(M, K) * Kp);
    if (codes_itself(M, K) || linear_in_tiles(M, N, K, source == DSS_TOKENS_MAP)) return 0;
    return weights + align256(M * Kp) + align256(M * 4);
}

}  // namespace

dss_status check_room(int64_t need, const void* workspace, int64_t workspace_bytes) {
    if (need == 0) return DSS_OK;
    if (!workspace || ((uintptr_t)workspace & 255u) != 0)
        return fail(DSS_E_INVALID, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < need)
        return fail(DSS_E_SHAPE, "workspace of %lld bytes is smaller than the %lld bytes needed",
                    (long long)workspace_bytes, (long long)need);
    return DSS_OK;
}

dss_status check_outputs(int64_t M, int32_t N, const void* out, dss_dtype out_dtype, int64_t out_token_stride,
                         int64_t out_channel_stride) {
    const bool rows = (out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1);
    const bool map = (out_token_stride == 1 || M <= 1) && (out_channel_stride >= M || N == 1);
    if (!rows && !map)
        return fail(out_channel_stride == 1 || out_token_stride == 1 ? DSS_E_INVALID : DSS_E_UNSUPPORTED,
                    "output strides %lld (tokens) and %lld (channels)", (long long)out_token_stride,
                    (long long)out_channel_stride);
    if (M > 0 && (!out || (uintptr_t)out % dtype_size(out_dtype) != 0))
        return fail(DSS_E_INVALID, "out is NULL or not aligned to its elements");
    return DSS_OK;
}

// The output's orientation: as rows where both would do.
bool is_map(int64_t M, int32_t N, int64_t out_token_stride, int64_t out_channel_stride) {
    return !((out_channel_stride == 1 || N == 1) && (out_token_stride >= N || M <= 1));
}

}  // namespace dss

extern "C" dss_status dss_tokens_workspace(int64_t M, int32_t N, int32_t K, dss_token_source source,
                                           int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (M < 0 || M > kMaxTokens || N < 1 || N > kMaxN || K < 1)
        return fail(DSS_E_INVALID, "%lld tokens of %d channels, %d outputs", (long long)M, K, N);
    if (source != DSS_TOKENS_ROWS && source != DSS_TOKENS_MAP && source != DSS_TOKENS_CODES)
        return fail(DSS_E_INVALID, "unknown token source %d", (int)source);
    if (K > kMaxK) return refuse_k(K);   // (what follows counts a row's bytes in 32 bits, and a layer's in 64)
    *workspace_bytes = workspace_bytes_of(M, N, K, source);
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
    s = check_room(workspace_bytes_of(M, N, K, DSS_TOKENS_CODES), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const int64_t ldo = map ? out_channel_stride : out_token_stride;
    const Layer L = {codes, codes_stride, scales, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out, ldo,
                     map, outputs_past(M, N, ldo, out, out_dtype)};
    hipError_t e = launch_matmul(L, out_dtype, false, static_cast<char*>(workspace), stream);
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
    const bool from_map = channel_stride != 1 && K > 1;
    s = check_room(workspace_bytes_of(M, N, K, from_map ? DSS_TOKENS_MAP : DSS_TOKENS_ROWS), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const bool map = is_map(M, N, out_token_stride, out_channel_stride);
    const int64_t ldo = map ? out_channel_stride : out_token_stride;
    Layer L = {nullptr, 0, nullptr, M, weight, weight_stride, weight_scales, N, K, bias, (int)act, out, ldo, map,
               outputs_past(M, N, ldo, out, out_dtype)};
    if (codes_itself(M, K) || linear_in_tiles(M, N, K, from_map)) {
        const Values V = {x, dtype, token_stride, channel_stride};
        hipError_t e = codes_itself(M, K) ? launch_linear_few(L, V, out_dtype, stream)
                                          : launch_linear_tiles(L, V, out_dtype, stream);
        return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
    }
    const int Kp = padded_k(K);
    char* room = static_cast<char*>(workspace);
    int8_t* codes = reinterpret_cast<int8_t*>(room) + (few_tokens(M, N, K) ? 0 : align256((int64_t)N * Kp));
    float* scales = reinterpret_cast<float*>(codes + align256(M * Kp));
    hipError_t e = launch_quantize_tokens(dtype, x, M, K, token_stride, channel_stride, codes, Kp, Kp, scales, stream);
    if (e != hipSuccess) return hip_fail(e, "quantize launch");
    L.codes = codes;
    L.codes_stride = Kp;
    L.scales = scales;
    e = launch_matmul(L, out_dtype, true, room, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "token product launch");
} catch (...) {
    return DSS_E_NOMEM;
}
