// Distillation from a teacher's top logits: with p = softmax(t / T) over a position's list and r = softmax(z / T)
// over all classes,
//   loss = s w T^2 sum_j p_j (log p_j - log r_{i_j}),   dloss / dz_c = s w T (r_c - sum_{j: i_j = c} p_j).
//
// Bound by memory: the logits are read and the gradient is written once.
//
// All exponents are taken to base 2 of differences to the largest logit, so that nothing
// overflows; logarithms of p and r come from those differences and the sums' logarithms.
#include <algorithm>
#include <cmath>

#include "dev_common.h"
#include "dss_internal.h"
#include "tokens.h"
#include "tokens_device.h"

namespace dss {

namespace {

constexpr int kMostTop = 1024;
constexpr int kThreads = 256;
constexpr float kLn2 = 0.69314718055994531f;
constexpr double kLog2e = 1.4426950408889634;

// What a call asks for.
struct Distill {
    const void* z;
    int64_t M, C, ts, cs;                // cs: the channels' stride
    const void* top;
    int top_bf16;
    int64_t top_ts, top_ps;
    const void* ids;
    int ids_64;
    int64_t ids_ts, ids_ps;
    int k;
    const float* weights;
    float to_log2;                       // log2(e) / T
    float scale, T;
    float* losses;
    void* grad;                          // NULL: the losses alone
    int64_t gts, gcs;
};

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }

// The class of place j: -1 for an empty place, C for one that there is not.
__device__ __forceinline__ int64_t class_of(const Distill& D, int64_t m, int j) {
    const int64_t at = m * D.ids_ts + j * D.ids_ps;
    const int64_t id = D.ids_64 ? static_cast<const int64_t*>(D.ids)[at] : (int64_t)static_cast<const int32_t*>(D.ids)[at];
    return id < 0 ? -1 : min(id, D.C);
}
__device__ __forceinline__ float teacher_of(const Distill& D, int64_t m, int j) {
    const int64_t at = m * D.top_ts + j * D.top_ps;
    return D.top_bf16 ? to_f32(static_cast<const uint16_t*>(D.top)[at]) : static_cast<const float*>(D.top)[at];
}

// Over a workgroup's threads.  `room` has a place for each wave; two calls in a row need a barrier between.
struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};
template <typename Op>
__device__ __forceinline__ float over_threads(float v, float* room) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = Op::of(v, __shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
    for (int w = 1; w < (int)blockDim.x / 64; ++w) v = Op::of(v, room[w]);
    return v;
}

// A workgroup for each position.
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_kernel(Distill D) {
    __shared__ float room[kThreads / 64];
    __shared__ float p[kMostTop];
    __shared__ int64_t ids[kMostTop];
    const int64_t m = blockIdx.x;
    const T* z = static_cast<const T*>(D.z) + m * D.ts;
    T* grad = static_cast<T*>(D.grad) + m * D.gts;
    const float weight = D.weights ? D.weights[m] : 1.f;
    constexpr int J = kMostTop / kThreads;
    float t[J], zj[J];
    int64_t id[J];
    float t_max = -INFINITY;
    int state = 0;                       // 1: a place that counts (a NaN does), 2: a class that there is not
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        id[n] = j < D.k ? class_of(D, m, j) : -1;
        t[n] = id[n] >= 0 ? teacher_of(D, m, j) : -INFINITY;
        zj[n] = id[n] >= 0 && id[n] < D.C ? to_f32(z[id[n] * D.cs]) : 0.f;
        state |= (t[n] != -INFINITY ? 1 : 0) | (id[n] >= D.C ? 3 : 0);
        t_max = fmaxf(t_max, t[n]);
    }
    t_max = over_threads<Max>(t_max, room);
    const bool wrong = __syncthreads_or(state & 2);
    if (!__syncthreads_or(state & 1) || weight == 0.f) {         // not to be learnt
        if (threadIdx.x == 0) D.losses[m] = 0.f;
        if (D.grad)
            for (int64_t c = threadIdx.x; c < D.C; c += kThreads) store_elem(grad + c * D.gcs, 0.f);
        return;
    }
    const float nan = wrong ? __uint_as_float(0x7fc00000u) : 0.f;
    float sum_p = 0.f;
#pragma unroll
    for (int n = 0; n < J; ++n) sum_p += t[n] == -INFINITY ? 0.f : exp2_of((t[n] - t_max) * D.to_log2);
    sum_p = over_threads<Sum>(sum_p, room) + nan;
    float z_max = -INFINITY;
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads) z_max = fmaxf(z_max, to_f32(z[c * D.cs]));
    z_max = over_threads<Max>(z_max, room);
    float sum_r = 0.f;
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads) sum_r += exp2_of((to_f32(z[c * D.cs]) - z_max) * D.to_log2);
    sum_r = over_threads<Sum>(sum_r, room);
    // log r - log p = (z - z_max - t + t_max) / T + log(sum_p / sum_r)
    const float log_sums = logf(sum_p) - logf(sum_r), per_T = D.to_log2 * kLn2;
    float loss = 0.f;
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        if (j >= D.k) continue;
        const float pj = (t[n] == -INFINITY ? 0.f : exp2_of((t[n] - t_max) * D.to_log2)) / sum_p;
        if (!(pj <= 0.f)) loss += pj * (((t[n] - t_max) - (zj[n] - z_max)) * per_T - log_sums);
        p[j] = pj;
        ids[j] = id[n];
    }
    loss = over_threads<Sum>(loss, room);    // (with barriers: p and ids are there)
    const float sw = D.scale * weight;
    if (threadIdx.x == 0) D.losses[m] = sw * D.T * (D.T * loss);
    if (!D.grad) return;
    const float g = sw * D.T, per_sum = 1.f / sum_r + nan;
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads)
        store_elem(grad + c * D.gcs, g * (exp2_of((to_f32(z[c * D.cs]) - z_max) * D.to_log2) * per_sum));
    __syncthreads();
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        if (j >= D.k || id[n] < 0 || id[n] >= D.C) continue;
        float of_class = 0.f;            // (a class may be there more than once)
        for (int i = 0; i < D.k; ++i) of_class += ids[i] == id[n] ? p[i] : 0.f;
        store_elem(grad + id[n] * D.gcs, g * (exp2_of((zj[n] - z_max) * D.to_log2) * per_sum - of_class));
    }
}

hipError_t launch_distill(const Distill& D, dss_dtype dt, hipStream_t s) {
    for (int64_t m = 0; m < D.M; m += kSlabTokens) {
        Distill S = D;
        S.M = std::min(D.M - m, kSlabTokens);
        const int64_t es = (int64_t)dtype_size(dt);
        S.z = static_cast<const char*>(D.z) + m * D.ts * es;
        S.top = static_cast<const char*>(D.top) + m * D.top_ts * (D.top_bf16 ? 2 : 4);
        S.ids = static_cast<const char*>(D.ids) + m * D.ids_ts * (D.ids_64 ? 8 : 4);
        if (D.weights) S.weights = D.weights + m;
        S.losses = D.losses + m;
        if (D.grad) S.grad = static_cast<char*>(D.grad) + m * D.gts * es;
        const dim3 grid((unsigned)S.M);
        if (dt == DSS_BF16) distill_kernel<uint16_t><<<grid, kThreads, 0, s>>>(S);
        else distill_kernel<float><<<grid, kThreads, 0, s>>>(S);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_distill_tokens(const void* logits, dss_dtype dtype, int64_t M, int32_t C, int64_t token_stride,
                                         int64_t channel_stride, const dss_top_logits* top, const float* token_weights,
                                         float temperature, float scale, float* losses, void* grad,
                                         int64_t grad_token_stride, int64_t grad_channel_stride, void* workspace,
                                         int64_t workspace_bytes, hipStream_t stream) try {
    using namespace dss;
    dss_status s = check_tokens(logits, dtype, M, C, token_stride, channel_stride);
    if (s != DSS_OK) return s;
    if (!top) return fail(DSS_E_INVALID, "NULL list of the teacher's logits");
    if (top->count < 1 || top->count > kMostTop)
        return fail(DSS_E_INVALID, "%d of the teacher's logits (1 to %d)", top->count, kMostTop);
    if (top->dtype != DSS_F32 && top->dtype != DSS_BF16) return fail(DSS_E_UNSUPPORTED, "unknown dtype %d of the teacher's logits", top->dtype);
    if (top->id_bytes != 4 && top->id_bytes != 8) return fail(DSS_E_UNSUPPORTED, "classes of %d bytes (4 or 8)", top->id_bytes);
    if (top->token_stride < 0 || top->place_stride < 0 || top->id_token_stride < 0 || top->id_place_stride < 0)
        return fail(DSS_E_INVALID, "negative stride of the teacher's lists");
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(scale))
        return fail(DSS_E_INVALID, "a temperature of %g and a scale of %g", (double)temperature, (double)scale);
    if (temperature < 0x1p-60f || temperature > 0x1p60f)
        return fail(DSS_E_UNSUPPORTED, "a temperature of %g", (double)temperature);
    const double to_log2 = kLog2e / (double)temperature;
    const bool map = channel_stride != 1 && C > 1;
    if (grad) {
        const bool rows_out = (grad_channel_stride == 1 || C == 1) && (grad_token_stride >= C || M <= 1);
        const bool map_out = (grad_token_stride == 1 || M <= 1) && (grad_channel_stride >= M || C == 1);
        if (map ? !map_out : !rows_out)
            return fail(DSS_E_INVALID, "gradient strides %lld (tokens) and %lld (channels) for logits of %lld and %lld",
                        (long long)grad_token_stride, (long long)grad_channel_stride, (long long)token_stride,
                        (long long)channel_stride);
        if ((uintptr_t)grad % dtype_size(dtype) != 0) return fail(DSS_E_INVALID, "grad is not aligned to its elements");
    }
    if (M == 0) return DSS_OK;
    if (!top->logits || (uintptr_t)top->logits % dtype_size((dss_dtype)top->dtype) != 0 || !top->ids ||
        (uintptr_t)top->ids % (unsigned)top->id_bytes != 0)
        return fail(DSS_E_INVALID, "the teacher's logits or classes are NULL or not aligned to their elements");
    if (!losses || (uintptr_t)losses % 4 != 0 || (uintptr_t)token_weights % 4 != 0)
        return fail(DSS_E_INVALID, "losses is NULL, or the losses or the weights are not aligned");
    s = check_room(DSS_DISTILL_WORKSPACE_BYTES, workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const Distill D = {logits, M, C, token_stride, channel_stride, top->logits, top->dtype == DSS_BF16, top->token_stride,
                       top->place_stride, top->ids, top->id_bytes == 8, top->id_token_stride, top->id_place_stride,
                       top->count, token_weights, (float)to_log2, scale, temperature, losses, grad, grad_token_stride,
                       grad_channel_stride};
    hipError_t e = launch_distill(D, dtype, stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "distillation launch");
} catch (...) {
    return DSS_E_NOMEM;
}
