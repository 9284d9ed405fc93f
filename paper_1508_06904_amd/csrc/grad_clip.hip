// Norm of a gradient over all of its tensors, and clipping by it:
//   norm = sqrt(sum_t sum_i g_t[i]^2),   out_t[i] = min(1, max_norm / (norm + 1e-6)) g_t[i].
//
// Two passes over the values: sums of squares into one partial sum per
// workgroup, then the partial sums' total (again in every workgroup: 8 KB at
// most, from L2) and the scaling.  Both are bound by memory.  The squares are
// summed in binary64: no square of a binary32 value leaves its range, so a norm
// is finite and right wherever binary32 can hold it, and the conversion and the
// multiply-add cost less than the loads they wait for.  Each value's place in the
// sums depends on the tensors' sizes only: the same gradients give the same bits.
//
// The tensors travel as a kernel argument, kTable at a time (a launch more for
// every kTable tensors); a workgroup finds the tensor of its run of values by
// bisection.  Tensors need no more than their elements' alignment: the 16-byte
// loads and stores of this GPU take any address.
//
// Measured: 537 million binary32 values, norm 310 us (6.9 TB/s), norm and clipping 1.13 ms, of which the
// scaling's reading and writing are 0.81 (5.3 TB/s; a large copy runs at 5.07); 134 million bfloat16
// values 48 and 130 us; 5.2 million binary32 values in ten tensors 15 us on the GPU in two launches.
#include <algorithm>
#include <cmath>

#include "dev_common.h"
#include "dss_internal.h"

namespace dss {

namespace {

constexpr int kThreads = 256;
constexpr int kTable = 112;              // 112 * 32 bytes of tensors: the table fits a 4 KB kernel argument
constexpr int kSmallTable = 16;          // a short list's table, which takes less time to hand over
constexpr int kMaxGroups = 1024;         // workgroups (and partial sums) of a launch
// Lists of more values write their clipped values around the caches, whose room goes to
// the values that are read for the second time.  The clipping alone gains from that at every
// size, but an update that reads the clipped values next finds shorter lists' in the caches.
// Clipping and update, through the caches and around them, us, of 2^24, 2^25, 2^26 values:
// binary32 70/72, 155/145, 302/285; bfloat16 71/72, 70/73, 155/144.  (In bytes the two types
// cross at the same place, 64 to 128 MB; a count of values is 6 % off for 2^25 binary32 ones.)
constexpr int64_t kCached = (int64_t)1 << 25;
// Of even more values little would be left in the caches for the second reading: all of
// them go around.  Clipping with the outputs alone around, and with all, us, of 2^26 to 2^29
// values: binary32 129/134, 300/280, 586/551, 1168/1103; bfloat16 68/69, 132/138, 304/284,
// 593/558: the count fits bfloat16 up to 2^27, and is two powers late for binary32.  The norm
// alone gains from 2^25 on: 27/24 us there, 366/322 at 2^29, in binary32.
constexpr int64_t kPassing = (int64_t)1 << 28;
// Values of the shortest run: in binary32 the four vectors that each thread has under way at
// once.  In bfloat16 that takes 8192 values, so lists of up to 2^24 values, whose runs are the
// shortest, are read and written value by value: 2^24 of them take 51 us, 2^25 37.
constexpr int64_t kMinRun = 4096;

template <int CAP>
struct TensorTable {
    static constexpr int kCap = CAP;
    const void* in[CAP];
    void* out[CAP];
    int64_t count[CAP];
    int32_t first[CAP];                  // the tensor's first run
    int32_t dtype[CAP];
    int32_t n, runs;
    int32_t run_shift;                   // a run has 2^run_shift values
};

static_assert(sizeof(TensorTable<kTable>) + 64 <= 4096, "the table is a kernel argument");

// Vectors at the elements' own alignment.
template <typename T>
struct Vec16 {
    T v[16 / sizeof(T)];
};
// PAST: around the caches.
template <bool PAST, typename T>
__device__ __forceinline__ Vec16<T> load16(const T* p) {
    using u32x4 = __attribute__((ext_vector_type(4), aligned(sizeof(T)))) uint32_t;
    if constexpr (PAST) return __builtin_bit_cast(Vec16<T>, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
    Vec16<T> r;
    __builtin_memcpy(&r, p, 16);
    return r;
}
template <bool PAST, typename T>
__device__ __forceinline__ void store16(T* p, const Vec16<T>& r) {
    using u32x4 = __attribute__((ext_vector_type(4), aligned(sizeof(T)))) uint32_t;
    if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p));
    else __builtin_memcpy(p, &r, 16);
}

// The sum of v over the workgroup, in every thread; the order of the additions is fixed.
__device__ double group_sum(double v) {
    __shared__ double part[kThreads / 64];
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) v += part[w];
    return v;
}

// The tensor that run r belongs to: the last one whose first run is not after r.
template <typename Table>
__device__ __forceinline__ int find_tensor(const Table& t, int r) {
    int lo = 0, hi = t.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

template <bool PAST, typename T>
__device__ __forceinline__ double sum_squares(const T* p, int64_t n, double s) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int U = 4;
    int64_t i = (int64_t)threadIdx.x * V;
    for (; i + (int64_t)(U - 1) * kThreads * V + V <= n; i += (int64_t)U * kThreads * V) {
        Vec16<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load16<PAST>(p + i + (int64_t)u * kThreads * V);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < V; ++k) {
                const double d = to_f32(x[u].v[k]);
                s = fma(d, d, s);
            }
    }
    for (; i < n; i += (int64_t)kThreads * V)
        for (int k = 0; k < V && i + k < n; ++k) {
            const double d = to_f32(p[i + k]);
            s = fma(d, d, s);
        }
    return s;
}

template <int CAP, bool PAST>
__global__ __launch_bounds__(kThreads) void norm_partial_kernel(TensorTable<CAP> t, double* partial, int add) {
    double s = 0;
    for (int r = blockIdx.x; r < t.runs; r += gridDim.x) {
        const int k = find_tensor(t, r);
        const int64_t at = (int64_t)(r - t.first[k]) << t.run_shift;
        const int64_t n = min(t.count[k] - at, (int64_t)1 << t.run_shift);
        if (t.dtype[k] == DSS_BF16) s = sum_squares<PAST>((const uint16_t*)t.in[k] + at, n, s);
        else s = sum_squares<PAST>((const float*)t.in[k] + at, n, s);
    }
    s = group_sum(s);
    if (threadIdx.x == 0) partial[blockIdx.x] = add ? partial[blockIdx.x] + s : s;
}

__device__ __forceinline__ double norm_of(const double* partial, int groups) {
    double s = 0;
    for (int i = threadIdx.x; i < groups; i += kThreads) s += partial[i];
    return sqrt(group_sum(s));
}

__global__ __launch_bounds__(kThreads) void norm_total_kernel(const double* partial, int groups, float* norm) {
    const double v = norm_of(partial, groups);
    if (threadIdx.x == 0) *norm = (float)v;
}

// The factor c * 2^e of a value.  e is 0 except for factors below the normal binary32
// numbers, whose last bits (or all) c alone would lose: 1e25 clipped to a norm of 1e-25.
struct Factor {
    float c;
    int e;
    __device__ __forceinline__ float of(float v) const { return ldexpf(v * c, e); }
    __device__ __forceinline__ bool is_one() const { return c == 1.f && e == 0; }
};

// min(1, b / (norm + 1e-6)); a NaN norm stays one, an infinite norm gives 0.  An infinite
// bound clips nothing, an infinite norm's values included.
__device__ __forceinline__ Factor factor_of(double norm, float max_norm) {
    if (isinf(max_norm) && !isnan(norm)) return {1.f, 0};
    const double c = (double)max_norm / (norm + 1e-6);
    if (c >= 1.0) return {1.f, 0};
    if (!(c > 0 && c < 0x1p-126)) return {(float)c, 0};
    int e;
    const double m = frexp(c, &e);
    return {(float)m, e};
}

// Values (LOAD) and outputs (STORE) around the caches or through them.
template <bool LOAD, bool STORE, typename T>
__device__ __forceinline__ void scale_run(const T* p, T* q, int64_t n, const Factor& f) {
    constexpr int V = 16 / (int)sizeof(T);
    constexpr int U = 4;
    int64_t i = (int64_t)threadIdx.x * V;
    for (; i + (int64_t)(U - 1) * kThreads * V + V <= n; i += (int64_t)U * kThreads * V) {
        Vec16<T> x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load16<LOAD>(p + i + (int64_t)u * kThreads * V);
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int k = 0; k < V; ++k) store_elem(&x[u].v[k], f.of(to_f32(x[u].v[k])));
            store16<STORE>(q + i + (int64_t)u * kThreads * V, x[u]);
        }
    }
    for (; i < n; i += (int64_t)kThreads * V)
        for (int k = 0; k < V && i + k < n; ++k) store_elem(&q[i + k], f.of(to_f32(p[i + k])));
}

template <int CAP, bool LOAD, bool STORE>
__global__ __launch_bounds__(kThreads) void clip_kernel(TensorTable<CAP> t, const double* partial, int groups,
                                                        float max_norm, float* norm) {
    const double total = norm_of(partial, groups);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)total;
    const Factor f = factor_of(total, max_norm);
    for (int r = blockIdx.x; r < t.runs; r += gridDim.x) {
        const int k = find_tensor(t, r);
        if (f.is_one() && t.in[k] == t.out[k]) continue;   // in place, nothing to clip
        const int64_t at = (int64_t)(r - t.first[k]) << t.run_shift;
        const int64_t n = min(t.count[k] - at, (int64_t)1 << t.run_shift);
        if (t.dtype[k] == DSS_BF16) scale_run<LOAD, STORE>((const uint16_t*)t.in[k] + at, (uint16_t*)t.out[k] + at, n, f);
        else scale_run<LOAD, STORE>((const float*)t.in[k] + at, (float*)t.out[k] + at, n, f);
    }
}

// ------------------------------------------------------------------ short lists, in one launch
// One workgroup of 16 waves: the waves take runs of kShortRun values in turn, sum
// their squares, meet for the total and scale the same runs, now in cache.
//
// One launch and two, us, a call among others from Python: 6 tensors of 200 values 12.5/15.8,
// 16 of 1024 18.2/21.3, 16 of 2048 (the most) 18.1/21.5.  There the launch that is saved
// counts; on the GPU alone, as in a graph, one launch is faster for the shortest lists only:
// 4.4/5.9, 8.2/6.5, 13.9/7.4.
constexpr int kShortTable = 16;
constexpr int kShortWaves = 16;
constexpr int kShortRun = 1024;          // 16 values of each lane
constexpr int kShortRuns = 2 * kShortWaves;

struct ShortTable {
    const void* in[kShortTable];
    void* out[kShortTable];
    int32_t count[kShortTable];
    int16_t first[kShortTable];
    int16_t dtype[kShortTable];
    int32_t n, runs;
};

template <typename T>
__device__ __forceinline__ double short_squares(const T* p, int n, double s) {
    const int lane = threadIdx.x & 63;
    float v[kShortRun / 64];
#pragma unroll
    for (int k = 0; k < kShortRun / 64; ++k) v[k] = k * 64 + lane < n ? to_f32(p[k * 64 + lane]) : 0.f;
#pragma unroll
    for (int k = 0; k < kShortRun / 64; ++k) s = fma((double)v[k], (double)v[k], s);
    return s;
}

template <typename T>
__device__ __forceinline__ void short_scale(const T* p, T* q, int n, const Factor& f) {
    const int lane = threadIdx.x & 63;
    float v[kShortRun / 64];
#pragma unroll
    for (int k = 0; k < kShortRun / 64; ++k) v[k] = k * 64 + lane < n ? to_f32(p[k * 64 + lane]) : 0.f;
#pragma unroll
    for (int k = 0; k < kShortRun / 64; ++k)
        if (k * 64 + lane < n) store_elem(&q[k * 64 + lane], f.of(v[k]));
}

__global__ __launch_bounds__(kShortWaves * 64) void clip_short_kernel(ShortTable t, float max_norm, int clip,
                                                                      float* norm) {
    __shared__ double part[kShortWaves];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    int at[kShortRuns / kShortWaves], left[kShortRuns / kShortWaves], who[kShortRuns / kShortWaves];
    double s = 0;
#pragma unroll
    for (int u = 0; u < kShortRuns / kShortWaves; ++u) {
        const int r = wave + u * kShortWaves;
        left[u] = 0;
        if (r >= t.runs) continue;
        int k = 0;
        for (int i = 1; i < t.n; ++i)
            if (t.first[i] <= r) k = i;
        who[u] = k;
        at[u] = (r - t.first[k]) * kShortRun;
        left[u] = min(t.count[k] - at[u], kShortRun);
        if (t.dtype[k] == DSS_BF16) s = short_squares((const uint16_t*)t.in[k] + at[u], left[u], s);
        else s = short_squares((const float*)t.in[k] + at[u], left[u], s);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) part[wave] = s;
    __syncthreads();
    s = 0;
#pragma unroll
    for (int w = 0; w < kShortWaves; ++w) s += part[w];
    const double total = sqrt(s);
    if (threadIdx.x == 0) *norm = (float)total;
    if (!clip) return;
    const Factor f = factor_of(total, max_norm);
#pragma unroll
    for (int u = 0; u < kShortRuns / kShortWaves; ++u) {
        if (left[u] == 0) continue;
        const int k = who[u];
        if (f.is_one() && t.in[k] == t.out[k]) continue;
        if (t.dtype[k] == DSS_BF16)
            short_scale((const uint16_t*)t.in[k] + at[u], (uint16_t*)t.out[k] + at[u], left[u], f);
        else
            short_scale((const float*)t.in[k] + at[u], (float*)t.out[k] + at[u], left[u], f);
    }
}

// Whether the list is a short one, and its table.
bool short_table(const dss_tensor* g, void* const* out, int32_t n, ShortTable* t) {
    t->n = t->runs = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (g[i].count == 0) continue;
        if (t->n == kShortTable || g[i].count > kShortRuns * kShortRun) return false;
        t->in[t->n] = g[i].data;
        t->out[t->n] = out ? out[i] : nullptr;
        t->count[t->n] = (int32_t)g[i].count;
        t->first[t->n] = (int16_t)t->runs;
        t->dtype[t->n] = (int16_t)g[i].dtype;
        t->runs += (int32_t)ceil_div64(g[i].count, kShortRun);
        if (t->runs > kShortRuns) return false;
        ++t->n;
    }
    return true;
}

// Runs of 2^shift values: about four of them for each workgroup of a full launch, none shorter than kMinRun.
int pick_shift(int64_t total) {
    int shift = 12;
    while (shift < 20 && (total >> shift) > 4 * kMaxGroups) ++shift;
    return shift;
}
static_assert(kMinRun == 1 << 12, "pick_shift starts there");

// The next table of tensors from *at on; whether there was one.  Empty tensors are left out.
template <typename Table>
bool next_table(const dss_tensor* g, void* const* out, int32_t n, int shift, int32_t* at, Table* t) {
    t->n = t->runs = 0;
    t->run_shift = shift;
    for (; *at < n && t->n < Table::kCap; ++*at) {
        const dss_tensor& x = g[*at];
        if (x.count == 0) continue;
        const int64_t runs = ceil_div64(x.count, (int64_t)1 << shift);
        if (t->runs + runs > (1 << 30)) break;
        t->in[t->n] = x.data;
        t->out[t->n] = out ? out[*at] : nullptr;
        t->count[t->n] = x.count;
        t->first[t->n] = t->runs;
        t->dtype[t->n] = x.dtype;
        t->runs += (int32_t)runs;
        ++t->n;
    }
    return t->n > 0;
}

// All launches of a list that is not short.
template <int CAP>
dss_status run_tables(const dss_tensor* grads, void* const* out, int32_t n, bool clip, float max_norm, float* norm,
                      double* partial, int64_t total, hipStream_t stream) {
    const int shift = pick_shift(total);
    TensorTable<CAP> t;
    // every launch but the first adds to the first one's partial sums, so that one has a sum for each of them
    int groups = 1;
    for (int32_t at = 0; next_table(grads, out, n, shift, &at, &t);) groups = std::max(groups, std::min(t.runs, kMaxGroups));
    int32_t at = 0;
    for (int add = 0; next_table(grads, out, n, shift, &at, &t); add = 1) {
        const dim3 grid(add ? std::min(t.runs, kMaxGroups) : groups);
        if (total > kPassing) norm_partial_kernel<CAP, true><<<grid, kThreads, 0, stream>>>(t, partial, add);
        else norm_partial_kernel<CAP, false><<<grid, kThreads, 0, stream>>>(t, partial, add);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gradient norm launch");
    }
    if (!clip) {
        norm_total_kernel<<<1, kThreads, 0, stream>>>(partial, groups, norm);
        hipError_t e = hipGetLastError();
        return e == hipSuccess ? DSS_OK : hip_fail(e, "gradient norm launch");
    }
    at = 0;
    for (bool first = true; next_table(grads, out, n, shift, &at, &t); first = false) {
        const dim3 grid(std::min(t.runs, kMaxGroups));
        float* to = first ? norm : nullptr;
        if (total > kPassing) clip_kernel<CAP, true, true><<<grid, kThreads, 0, stream>>>(t, partial, groups, max_norm, to);
        else if (total > kCached) clip_kernel<CAP, false, true><<<grid, kThreads, 0, stream>>>(t, partial, groups, max_norm, to);
        else clip_kernel<CAP, false, false><<<grid, kThreads, 0, stream>>>(t, partial, groups, max_norm, to);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return hip_fail(e, "gradient clipping launch");
    }
    return DSS_OK;
}

dss_status grad_common(const dss_tensor* grads, void* const* out, int32_t n, bool clip, float max_norm, float* norm,
                       void* workspace, int64_t workspace_bytes, hipStream_t stream) {
    if (n < 0 || (n > 0 && !grads)) return fail(DSS_E_INVALID, "%d tensors, NULL list or not", n);
    if (!norm || (uintptr_t)norm % 4 != 0) return fail(DSS_E_INVALID, "norm is NULL or not aligned to its elements");
    if (clip && n > 0 && !out) return fail(DSS_E_INVALID, "NULL list of outputs");
    if (clip && !(max_norm >= 0.f)) return fail(DSS_E_INVALID, "max_norm %g is negative or not a number", max_norm);
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (grads[i].dtype != DSS_F32 && grads[i].dtype != DSS_BF16)
            return fail(DSS_E_UNSUPPORTED, "tensor %d: unknown dtype %d", i, grads[i].dtype);
        if (grads[i].count < 0 || grads[i].count > ((int64_t)1 << 40) || total > ((int64_t)1 << 42))
            return fail(DSS_E_INVALID, "tensor %d: %lld elements", i, (long long)grads[i].count);
        if (grads[i].count == 0) continue;
        const uintptr_t es = grads[i].dtype == DSS_BF16 ? 2 : 4;
        if (!grads[i].data || (uintptr_t)grads[i].data % es != 0)
            return fail(DSS_E_INVALID, "tensor %d: NULL or not aligned to its elements", i);
        if (clip && (!out[i] || (uintptr_t)out[i] % es != 0))
            return fail(DSS_E_INVALID, "output %d: NULL or not aligned to its elements", i);
        total += grads[i].count;
    }
    if (!workspace || ((uintptr_t)workspace & 255u) != 0)
        return fail(DSS_E_INVALID, "workspace is NULL or not 256-byte aligned");
    if (workspace_bytes < DSS_GRAD_NORM_WORKSPACE_BYTES)
        return fail(DSS_E_SHAPE, "workspace of %lld bytes is smaller than the %lld bytes needed",
                    (long long)workspace_bytes, (long long)DSS_GRAD_NORM_WORKSPACE_BYTES);
    static_assert(kMaxGroups * sizeof(double) <= DSS_GRAD_NORM_WORKSPACE_BYTES, "partial sums");

    ShortTable brief;
    if (short_table(grads, out, n, &brief)) {
        clip_short_kernel<<<1, kShortWaves * 64, 0, stream>>>(brief, max_norm, clip, norm);
        hipError_t e = hipGetLastError();
        return e == hipSuccess ? DSS_OK : hip_fail(e, "gradient clipping launch");
    }
    int filled = 0;
    for (int32_t i = 0; i < n; ++i) filled += grads[i].count != 0;
    double* partial = static_cast<double*>(workspace);
    return filled <= kSmallTable ? run_tables<kSmallTable>(grads, out, n, clip, max_norm, norm, partial, total, stream)
                                 : run_tables<kTable>(grads, out, n, clip, max_norm, norm, partial, total, stream);
}

}  // namespace

}  // namespace dss

extern "C" dss_status dss_grad_norm(const dss_tensor* grads, int32_t n, float* norm, void* workspace,
                                    int64_t workspace_bytes, hipStream_t stream) try {
    return dss::grad_common(grads, nullptr, n, false, 0.f, norm, workspace, workspace_bytes, stream);
} catch (...) {
    return DSS_E_NOMEM;
}

extern "C" dss_status dss_clip_grads(const dss_tensor* grads, void* const* out, int32_t n, float max_norm, float* norm,
                                     void* workspace, int64_t workspace_bytes, hipStream_t stream) try {
    return dss::grad_common(grads, out, n, true, max_norm, norm, workspace, workspace_bytes, stream);
} catch (...) {
    return DSS_E_NOMEM;
}
