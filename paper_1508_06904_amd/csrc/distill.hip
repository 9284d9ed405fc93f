// Distillation from a teacher's top logits: with p = softmax(t / T) over a position's list and r = softmax(z / T)
// over all classes,
//   loss = s w T^2 sum_j p_j (log p_j - log r_{i_j}),   dloss / dz_c = s w T (r_c - sum_{j: i_j = c} p_j).
//
// Bound by memory: the logits are read and the gradient is written once.  This file has the entry point
// and the rows (a position's classes adjacent), distill_map.hip the maps.
//
// 4096 rows of 32768 bfloat16 classes: 105 us, 5.1 TB/s; the loss alone of 513 rows of 131071 binary32 classes 48 us (parts 43, 6.3 TB/s);
// one row of 4 classes 3 us.
#include <algorithm>
#include <cmath>

#include "dev_common.h"
#include "distill.h"
#include "dss_internal.h"

namespace dss {

namespace {

constexpr int kThreads = 256;
constexpr double kLog2e = 1.4426950408889634;

// ------------------------------------------------------------------ any strides
// A workgroup for each position, which reads its logits three times: maps of more than 128 classes with lists of more than 128 places.
// (Neighbours, which share lines, on one XCD: 20000 positions of 1000 classes 397 us for 932.)
template <typename T>
__global__ __launch_bounds__(kThreads) void distill_kernel(Distill D) {
    __shared__ float room[kThreads / 64 * 2];
    __shared__ float p[kMostTop];
    __shared__ int ids[kMostTop];
    const int64_t m = xcd_order(blockIdx.x, gridDim.x);
    const T* z = static_cast<const T*>(D.z) + m * D.ts;
    T* grad = static_cast<T*>(D.grad) + m * D.gts;
    const float weight = D.weights ? D.weights[m] : 1.f;
    constexpr int J = kMostTop / kThreads;
    Place a[J];
    float lists[2] = {-INFINITY, 0.f};
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        a[n] = j < D.k ? place_of(D, m, j, z) : Place{-1, -INFINITY, 0.f};
        lists[0] = fmaxf(lists[0], a[n].t);
        lists[1] = fmaxf(lists[1], a[n].state(D));
    }
    over_lanes<Max, kThreads>(lists, room);
    const float t_max = lists[0];
    if (weight == 0.f || lists[1] == 0.f) {                      // not to be learnt
        if (threadIdx.x == 0) D.losses[m] = 0.f;
        if (D.grad)
            for (int64_t c = threadIdx.x; c < D.C; c += kThreads) store_elem(grad + c * D.gcs, 0.f);
        return;
    }
    const float nan = lists[1] == 3.f ? quiet_nan() : 0.f;
    float z_max[1] = {-INFINITY};
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads) z_max[0] = fmaxf(z_max[0], to_f32(z[c * D.cs]));
    over_lanes<Max, kThreads>(z_max, room);
    float sums[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < J; ++n) sums[0] += weight_of(D, a[n].t, t_max);
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads) sums[1] += exp2_of((to_f32(z[c * D.cs]) - z_max[0]) * D.to_log2);
    over_lanes<Sum, kThreads>(sums, room);
    const float sum_p = sums[0] + nan, sum_r = sums[1] + nan, log_sums = logf(sum_p) - logf(sum_r);
    float loss[1] = {0.f};
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        if (j >= D.k) continue;
        p[j] = weight_of(D, a[n].t, t_max) / sum_p;
        ids[j] = a[n].id;
        loss[0] += loss_of(D, p[j], a[n].t, t_max, a[n].z, z_max[0], log_sums);
    }
    over_lanes<Sum, kThreads>(loss, room);   // (with barriers: p and ids are there)
    const float sw = D.scale * weight;
    if (threadIdx.x == 0) D.losses[m] = sw * D.T * (D.T * loss[0]);
    if (!D.grad) return;
    const float g = sw * D.T, per_sum = 1.f / sum_r;
    for (int64_t c = threadIdx.x; c < D.C; c += kThreads)
        store_elem(grad + c * D.gcs, g * (exp2_of((to_f32(z[c * D.cs]) - z_max[0]) * D.to_log2) * per_sum));
    __syncthreads();
#pragma unroll
    for (int n = 0; n < J; ++n) {
        const int j = n * kThreads + threadIdx.x;
        if (j >= D.k || a[n].id < 0 || a[n].id >= (int)D.C) continue;
        float of_class = 0.f;            // (a class may be there more than once)
        for (int i = 0; i < D.k; ++i) of_class += ids[i] == a[n].id ? p[i] : 0.f;
        store_elem(grad + a[n].id * D.gcs, g * (exp2_of((a[n].z - z_max[0]) * D.to_log2) * per_sum - of_class));
    }
}

// ------------------------------------------------------------------ rows
// A position's list in LDS: the teacher's logits (then p), the student's, and the classes.
struct List {
    float *t, *z;
    int* id;

    static __host__ __device__ size_t bytes(int k) { return (size_t)k * 12; }
    __device__ __forceinline__ List(char* lds, int k) : t((float*)lds), z(t + k), id((int*)(z + k)) {}
    // The sum of p over the places of a class, in the places' order.
    __device__ __forceinline__ float of_class(int c, int k) const {
        float s = 0.f;
        for (int i = 0; i < k; ++i) s += id[i] == c ? t[i] : 0.f;
        return s;
    }
};

// LPR threads hold a position's logits, CH chunks each, in registers: they are read once.
template <typename T, int LPR, int CH, bool PAST>
__global__ __launch_bounds__(LPR < kThreads ? kThreads : LPR) void distill_rows_kernel(Distill D) {
    constexpr int E = Logits<T>::E, ROWS = LPR < kThreads ? kThreads / LPR : 1;
    __shared__ float room[LPR > 64 ? LPR / 64 * 3 : 1];
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x % LPR, row = threadIdx.x / LPR, k = D.k;
    const int64_t m_own = (int64_t)blockIdx.x * ROWS + row, m = min(m_own, D.M - 1);
    const T* z = static_cast<const T*>(D.z) + m * D.ts;
    const float weight = D.weights ? D.weights[m] : 1.f;
    const List list(lds + row * List::bytes(k), k);
    Logits<T> c[CH];
    const int C = weight == 0.f ? 0 : (int)D.C, last = C / E;    // the chunk that C ends in, if it ends in one
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        c[i].clear();
        if (i * LPR + lane < last) c[i].template load<PAST>(z + (i * LPR + lane) * E);
    }
    if (C % E != 0 && last % LPR == lane) {
        Logits<T> end;
        end.load(z + last * E, C % E);
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (i == last / LPR) c[i] = end;
    }
    float tops[3] = {-INFINITY, 0.f, -INFINITY};       // of the list, its state, of the logits
    for (int j = lane; j < k; j += LPR) {
        const Place a = place_of(D, m, j, z);
        list.t[j] = a.t;
        list.z[j] = a.z;
        list.id[j] = a.id;
        tops[0] = fmaxf(tops[0], a.t);
        tops[1] = fmaxf(tops[1], a.state(D));
    }
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        tops[2] = c[i].top(tops[2]);
        c[i].forget();
    }
    over_lanes<Max, LPR>(tops, room);
    const float t_max = tops[0], z_max = tops[2];
    const bool live = weight != 0.f && tops[1] != 0.f;
    const float nan = tops[1] == 3.f ? quiet_nan() : 0.f;
    float sums[2] = {0.f, 0.f};
    for (int j = lane; j < k; j += LPR) sums[0] += weight_of(D, list.t[j], t_max);
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const float v = exp2_of((c[i].value(e) - z_max) * D.to_log2);
            if constexpr (sizeof(T) == 4) c[i].w[e] = __float_as_uint(v);     // (bfloat16 has no room for it)
            part += v;
        }
        sums[1] += part;
        c[i].forget();
    }
    over_lanes<Sum, LPR>(sums, room);
    const float sum_p = sums[0] + nan, sum_r = sums[1] + nan, log_sums = logf(sum_p) - logf(sum_r);
    float loss[1] = {0.f};
    for (int j = lane; j < k; j += LPR) {
        const float t = list.t[j], p = weight_of(D, t, t_max) / sum_p;
        loss[0] += loss_of(D, p, t, t_max, list.z[j], z_max, log_sums);
        list.t[j] = p;
    }
    over_lanes<Sum, LPR>(loss, room);
    const float sw = D.scale * weight;
    if (lane == 0 && m_own < D.M) D.losses[m] = live ? sw * D.T * (D.T * loss[0]) : 0.f;
    if (!D.grad) return;
    const float g = sw * D.T, per_sum = 1.f / sum_r, per = g * per_sum;
    T* grad = static_cast<T*>(D.grad) + m * D.gts;
    if (m_own < D.M) {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = (i * LPR + lane) * E;
            if (at >= (int)D.C) continue;
            float v[E] = {};
            if (live)
#pragma unroll
                for (int e = 0; e < E; ++e) v[e] = (sizeof(T) == 4 ? c[i].value(e) : exp2_of((c[i].value(e) - z_max) * D.to_log2)) * per;
            store_gradients<PAST>(grad + at, v, D.C - at);
        }
    }
    __syncthreads();                     // the classes of the list are stored over
    if (m_own >= D.M || !live) return;
    for (int j = lane; j < k; j += LPR) {
        const int id = list.id[j];
        if (id >= 0 && id < (int)D.C)
            store_elem(grad + id, g * (exp2_of((list.z[j] - z_max) * D.to_log2) * per_sum - list.of_class(id, k)));
    }
}

constexpr int kOwnClasses = 32768;       // of rows that never have several workgroups

// Rows longer than the registers hold, or too long for one workgroup of few: `parts` workgroups share a position's classes.  First
// each takes its part's largest logit and sum.
template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads) void distill_parts_kernel(Distill D, int64_t per_part, Part* parts) {
    constexpr int E = Logits<T>::E, U = 8;
    __shared__ float room[kThreads / 64];
    const int64_t m = blockIdx.y, c0 = blockIdx.x * per_part, c1 = min(c0 + per_part, D.C);
    if (D.weights && D.weights[m] == 0.f) return;
    const T* z = static_cast<const T*>(D.z) + m * D.ts;
    Part own = {-INFINITY, 0.f};
    for (int64_t at = c0 + threadIdx.x * E; at < c1; at += U * kThreads * E) {
        Logits<T> c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u].template load<PAST>(z + at + u * kThreads * E, c1 - at - u * kThreads * E);
        float top = own.top;
#pragma unroll
        for (int u = 0; u < U; ++u) top = c[u].top(top);
        const float to = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) sum += exp2_of((c[u].value(e) - to) * D.to_log2);
        own.sum = own.sum * exp2_of((own.top - to) * D.to_log2) + sum;
        own.top = top;
    }
    float top[1] = {own.top};
    over_lanes<Max, kThreads>(top, room);
    float sum[1] = {joined(D, {top[0], 0.f}, own).sum};
    over_lanes<Sum, kThreads>(sum, room);
    if (threadIdx.x == 0) parts[m * gridDim.x + blockIdx.x] = {top[0], sum[0]};
}

// Then the loss (workgroups 0 of a position) and the gradient of their parts.
template <typename T, bool PAST>
__global__ __launch_bounds__(kThreads) void distill_finish_kernel(Distill D, int64_t per_part, const Part* parts, int n_parts,
                                                                  int with_loss) {
    constexpr int E = Logits<T>::E, U = 4;
    __shared__ float room[kThreads / 64 * 3];
    extern __shared__ __align__(16) char lds[];
    const int64_t m = blockIdx.y, c0 = blockIdx.x * per_part, c1 = min(c0 + per_part, D.C);
    const int k = D.k;
    const T* z = static_cast<const T*>(D.z) + m * D.ts;
    T* grad = static_cast<T*>(D.grad) + m * D.gts;
    const float weight = D.weights ? D.weights[m] : 1.f;
    const List list(lds, k);
    float tops[3] = {-INFINITY, 0.f, -INFINITY};
    for (int j = threadIdx.x; j < k; j += kThreads) {
        // (the student's logits of other parts may be their gradients already, if these are written over them)
        const int id = class_of(D, m, j);
        const bool own = id >= c0 && id < c1;
        list.id[j] = id;
        list.t[j] = id >= 0 ? teacher_of(D, m, j) : -INFINITY;
        list.z[j] = id >= 0 && id < (int)D.C && (own || (with_loss && blockIdx.x == 0)) ? to_f32(z[id]) : 0.f;
        tops[0] = fmaxf(tops[0], list.t[j]);
        tops[1] = fmaxf(tops[1], Place{id, list.t[j], 0.f}.state(D));
    }
    Part own = {-INFINITY, 0.f};
    if (weight != 0.f)
        for (int p = threadIdx.x; p < n_parts; p += kThreads) own = joined(D, own, parts[m * n_parts + p]);
    tops[2] = own.top;
    over_lanes<Max, kThreads>(tops, room);
    const float t_max = tops[0], z_max = tops[2];
    const bool live = weight != 0.f && tops[1] != 0.f;
    const float nan = tops[1] == 3.f ? quiet_nan() : 0.f;
    float sums[2] = {0.f, joined(D, {z_max, 0.f}, own).sum};
    for (int j = threadIdx.x; j < k; j += kThreads) sums[0] += weight_of(D, list.t[j], t_max);
    over_lanes<Sum, kThreads>(sums, room);
    // (a row of -infinities has the sum 0 here, and no softmax)
    const float sum_p = sums[0] + nan, sum_r = z_max == -INFINITY ? quiet_nan() : sums[1] + nan;
    const float log_sums = logf(sum_p) - logf(sum_r);
    float loss[1] = {0.f};
    for (int j = threadIdx.x; j < k; j += kThreads) {
        const float t = list.t[j], p = weight_of(D, t, t_max) / sum_p;
        loss[0] += loss_of(D, p, t, t_max, list.z[j], z_max, log_sums);
        list.t[j] = p;
    }
    over_lanes<Sum, kThreads>(loss, room);
    const float sw = D.scale * weight;
    if (threadIdx.x == 0 && blockIdx.x == 0 && with_loss) D.losses[m] = live ? sw * D.T * (D.T * loss[0]) : 0.f;
    if (!D.grad) return;
    const float g = sw * D.T, per_sum = 1.f / sum_r, per = g * per_sum;
    for (int64_t at = c0 + threadIdx.x * E; at < c1; at += U * kThreads * E) {
        Logits<T> c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u].template load<PAST>(z + at + u * kThreads * E, live ? c1 - at - u * kThreads * E : 0);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[E];
#pragma unroll
            for (int e = 0; e < E; ++e) v[e] = live ? exp2_of((c[u].value(e) - z_max) * D.to_log2) * per : 0.f;
            const int64_t from = at + u * kThreads * E;
            if (from < c1) store_gradients<PAST>(grad + from, v, c1 - from);
        }
    }
    __syncthreads();                     // the classes of the list are stored over
    if (!live) return;
    for (int j = threadIdx.x; j < k; j += kThreads) {
        const int id = list.id[j];
        if (id >= c0 && id < c1)
            store_elem(grad + id, g * (exp2_of((list.z[j] - z_max) * D.to_log2) * per_sum - list.of_class(id, k)));
    }
}

template <typename T, int LPR, int CH>
hipError_t run_rows(const Distill& D, hipStream_t s) {
    constexpr int ROWS = LPR < kThreads ? kThreads / LPR : 1;
    // Long rows go around the caches: 4096 of 32768 bfloat16 classes 119 us through them, 105 around.  (Shorter rows' loads share
    // lines: 1 million of 40 classes 91 us, 113 around.)
    const bool past = LPR >= kThreads && D.M * D.C * (int64_t)sizeof(T) > kLarge;
    const auto kern = past ? distill_rows_kernel<T, LPR, CH, (LPR >= kThreads)> : distill_rows_kernel<T, LPR, CH, false>;
    kern<<<dim3((unsigned)ceil_div64(D.M, ROWS)), ROWS * LPR, ROWS * List::bytes(D.k), s>>>(D);
    return hipGetLastError();
}

template <typename T>
hipError_t run_parts(const Distill& D, Part* parts, hipStream_t s) {
    // enough workgroups for the units, of at least some thousand classes each
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(1024 / D.M, D.C / 4096));
    const int64_t per_part = ceil_div64(ceil_div64(D.C, most), 64) * 64, n = ceil_div64(D.C, per_part);
    const int64_t bytes = D.M * D.C * (int64_t)sizeof(T);
    const auto first = bytes > (D.grad ? kNeverCached : kLarge) ? distill_parts_kernel<T, true> : distill_parts_kernel<T, false>;
    const auto finish = bytes > kLarge ? distill_finish_kernel<T, true> : distill_finish_kernel<T, false>;
    first<<<dim3((unsigned)n, (unsigned)D.M), kThreads, 0, s>>>(D, per_part, parts);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const bool over = D.grad == D.z;     // the losses need all of the logits first
    Distill L = D;
    if (over) L.grad = nullptr;
    if (over || !D.grad) {
        finish<<<dim3(1, (unsigned)D.M), kThreads, List::bytes(D.k), s>>>(L, D.C, parts, (int)n, 1);
        e = hipGetLastError();
        if (e != hipSuccess || !D.grad) return e;
    }
    finish<<<dim3((unsigned)n, (unsigned)D.M), kThreads, List::bytes(D.k), s>>>(D, per_part, parts, (int)n, !over);
    return hipGetLastError();
}

template <typename T>
hipError_t run_distill(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s) {
    constexpr int E = Logits<T>::E;
    // Several workgroups for a row beyond what one holds in registers; for the losses alone from half of that, and where few
    // rows leave units empty.  In microseconds for one workgroup and for several, with the gradient:
    //                 32768 binary32 classes   60000 bfloat16    120000 bfloat16
    //   8 rows               9 / 12               13 / 12            20 / 12
    //   60 rows              9 / 13               14 / 17            22 / 18
    //   120 rows            11 / 17               16 / 18            24 / 23
    // and the losses alone of 4000 rows: 81 / 91, 85 / 91 and 243 / 159.
    const int64_t one = 512 * 16 * E, most = D.grad ? (D.M < 128 ? 65536 : 2 * one) : one;
    static_assert(512 * 16 * E >= kOwnClasses);
    if (D.C > most) {
        // (a launch has 65535 workgroups along y)
        const int64_t slab = 4096;
        for (int64_t m = 0; m < D.M; m += slab) {
            const hipError_t e = run_parts<T>(positions(D, dt, m, std::min(D.M - m, slab)), parts, s);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    for (int64_t m = 0; m < D.M; m += kSlabTokens) {
        const Distill S = positions(D, dt, m, std::min(D.M - m, kSlabTokens));
        // As few threads and registers for a row as hold it, and the lists of their workgroup's rows in 48 KB of LDS: what is
        // left empty is rows that are not on their way.  4096 rows of 40000 bfloat16 classes 148 us on 512 threads, 290 on
        // 1024; 20000 rows of 10000 156 us in 8 chunks, 187 in 16.
        const int64_t rows = (int64_t)(48 * 1024 / List::bytes(D.k));
        hipError_t e;
        if (D.C <= 4 * 4 * E && rows >= 64) e = run_rows<T, 4, 4>(S, s);
        else if (D.C <= 16 * 4 * E && rows >= 16) e = run_rows<T, 16, 4>(S, s);
        else if (D.C <= 64 * 4 * E && rows >= 4) e = run_rows<T, 64, 4>(S, s);
        else if (D.C <= 256 * 4 * E) e = run_rows<T, 256, 4>(S, s);
        else if (D.C <= 256 * 8 * E) e = run_rows<T, 256, 8>(S, s);
        else if (D.C <= 256 * 16 * E) e = run_rows<T, 256, 16>(S, s);
        else if (D.C <= 512 * 16 * E) e = run_rows<T, 512, 16>(S, s);
        else e = run_rows<T, 1024, 16>(S, s);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_distill(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s) {
    if (D.cs == 1 || D.C == 1)
        return dt == DSS_BF16 ? run_distill<uint16_t>(D, dt, parts, s) : run_distill<float>(D, dt, parts, s);
    return launch_distill_map(D, dt, parts, s);
}

}  // namespace

// A workgroup for each position.
hipError_t launch_distill_any(const Distill& D, dss_dtype dt, hipStream_t s) {
    for (int64_t m = 0; m < D.M; m += kSlabTokens) {
        const Distill S = positions(D, dt, m, std::min(D.M - m, kSlabTokens));
        const dim3 grid((unsigned)S.M);
        if (dt == DSS_BF16) distill_kernel<uint16_t><<<grid, kThreads, 0, s>>>(S);
        else distill_kernel<float><<<grid, kThreads, 0, s>>>(S);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

Distill positions(const Distill& D, dss_dtype dt, int64_t m, int64_t n) {
    Distill S = D;
    const int64_t es = (int64_t)dtype_size(dt);
    S.M = n;
    S.z = static_cast<const char*>(D.z) + m * D.ts * es;
    S.top = static_cast<const char*>(D.top) + m * D.top_ts * (D.top_bf16 ? 2 : 4);
    S.ids = static_cast<const char*>(D.ids) + m * D.ids_ts * (D.ids_64 ? 8 : 4);
    if (D.weights) S.weights = D.weights + m;
    S.losses = D.losses + m;
    if (D.grad) S.grad = static_cast<char*>(D.grad) + m * D.gts * es;
    return S;
}

}  // namespace dss

namespace dss {
static int64_t distill_workspace(int32_t C, bool map) {
    return C > (map ? kColumns : kOwnClasses) ? DSS_DISTILL_WORKSPACE_BYTES : 0;
}
}  // namespace dss

extern "C" dss_status dss_distill_workspace(int32_t C, int32_t map, int64_t* workspace_bytes) try {
    using namespace dss;
    if (!workspace_bytes) return fail(DSS_E_INVALID, "NULL output");
    if (C < 1) return fail(DSS_E_INVALID, "%d classes", C);
    *workspace_bytes = distill_workspace(C, map != 0);
    return DSS_OK;
} catch (...) {
    return DSS_E_NOMEM;
}

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
    if (top->dtype != DSS_F32 && top->dtype != DSS_BF16)
        return fail(DSS_E_UNSUPPORTED, "unknown dtype %d of the teacher's logits", top->dtype);
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
        if (grad == logits && ((grad_token_stride != token_stride && M > 1) || (grad_channel_stride != channel_stride && C > 1)))
            return fail(DSS_E_INVALID, "a gradient over the logits with other strides");
        if ((uintptr_t)grad % dtype_size(dtype) != 0) return fail(DSS_E_INVALID, "grad is not aligned to its elements");
    }
    if (M == 0) return DSS_OK;
    if (!top->logits || (uintptr_t)top->logits % dtype_size((dss_dtype)top->dtype) != 0 || !top->ids ||
        (uintptr_t)top->ids % (unsigned)top->id_bytes != 0)
        return fail(DSS_E_INVALID, "the teacher's logits or classes are NULL or not aligned to their elements");
    if (!losses || (uintptr_t)losses % 4 != 0 || (uintptr_t)token_weights % 4 != 0)
        return fail(DSS_E_INVALID, "losses is NULL, or the losses or the weights are not aligned");
    s = check_room(distill_workspace(C, map), workspace, workspace_bytes);
    if (s != DSS_OK) return s;
    const Distill D = {logits, M, C, token_stride, channel_stride, top->logits, top->dtype == DSS_BF16, top->token_stride,
                       top->place_stride, top->ids, top->id_bytes == 8, top->id_token_stride, top->id_place_stride,
                       top->count, token_weights, (float)to_log2, scale, temperature, losses, grad, grad_token_stride,
                       grad_channel_stride};
    hipError_t e = launch_distill(D, dtype, static_cast<Part*>(workspace), stream);
    return e == hipSuccess ? DSS_OK : hip_fail(e, "distillation launch");
} catch (...) {
    return DSS_E_NOMEM;
}
