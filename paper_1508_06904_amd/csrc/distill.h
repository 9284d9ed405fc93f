// Internal declarations of the distillation from a teacher's top logits (distill.hip, distill_map.hip) and the device
// helpers that its kernels share.
//
// All exponents are taken to base 2 of differences to the largest logit, so that nothing
// overflows; logarithms of p and r come from those differences and the sums' logarithms.
#pragma once

#include "tokens.h"
#include "tokens_device.h"

namespace dss {

constexpr int kMostTop = 1024;
constexpr float kLn2 = 0.69314718055994531f;

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

// Bytes of logits beyond which a pass over them had better leave the caches to others; and beyond which the next pass
// would not find them there either.
constexpr int64_t kLarge = (int64_t)1 << 26, kNeverCached = (int64_t)1 << 28;

// The largest logit of a part of a position's classes, and the sum of exponentials of differences to it.
struct Part {
    float top, sum;
};

// The call from position m on, n positions.
Distill positions(const Distill& D, dss_dtype dt, int64_t m, int64_t n);

// Logits whose positions are adjacent.  `parts` has room for kMostParts.
constexpr int kMostParts = DSS_DISTILL_WORKSPACE_BYTES / (int)sizeof(Part);
constexpr int kColumns = 128;            // classes of a map that need no parts
hipError_t launch_distill_map(const Distill& D, dss_dtype dt, Part* parts, hipStream_t s);

// A workgroup for each position, any strides: maps with long lists.
hipError_t launch_distill_any(const Distill& D, dss_dtype dt, hipStream_t s);

__device__ __forceinline__ float exp2_of(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float quiet_nan() { return __uint_as_float(0x7fc00000u); }

// The class of place j: -1 for an empty place, C for one that there is not.
__device__ __forceinline__ int class_of(const Distill& D, int64_t m, int j) {
    const int64_t at = m * D.ids_ts + j * D.ids_ps;
    const int64_t id = D.ids_64 ? static_cast<const int64_t*>(D.ids)[at] : (int64_t)static_cast<const int32_t*>(D.ids)[at];
    return id < 0 ? -1 : (int)min(id, D.C);
}
__device__ __forceinline__ float teacher_of(const Distill& D, int64_t m, int j) {
    const int64_t at = m * D.top_ts + j * D.top_ps;
    return D.top_bf16 ? to_f32(static_cast<const uint16_t*>(D.top)[at]) : static_cast<const float*>(D.top)[at];
}

// A place of a list: its class (as class_of), the teacher's logit (-infinity for an empty place) and the student's.
struct Place {
    int id;
    float t, z;

    // 0: a place that does not count (of logit -infinity, whatever its class), 3: of a class that there is not, 1: any
    // other one (a NaN counts).
    __device__ __forceinline__ float state(const Distill& D) const { return t == -INFINITY ? 0.f : id >= (int)D.C ? 3.f : 1.f; }
};
template <typename T>
__device__ __forceinline__ Place place_of(const Distill& D, int64_t m, int j, const T* z) {
    Place r;
    r.id = class_of(D, m, j);
    r.t = r.id >= 0 ? teacher_of(D, m, j) : -INFINITY;
    r.z = r.id >= 0 && r.id < (int)D.C ? to_f32(z[r.id * D.cs]) : 0.f;
    return r;
}

// exp((t - t_max) / T) of a place, and its part of the loss: with p = that over sum_p,
// p (log p - log r) = p ((t - t_max) / T - (z - z_max) / T - log(sum_p / sum_r)).
__device__ __forceinline__ float weight_of(const Distill& D, float t, float t_max) {
    return t == -INFINITY ? 0.f : exp2_of((t - t_max) * D.to_log2);
}
__device__ __forceinline__ float loss_of(const Distill& D, float p, float t, float t_max, float z, float z_max, float log_sums) {
    return p <= 0.f ? 0.f : p * (((t - t_max) - (z - z_max)) * (D.to_log2 * kLn2) - log_sums);
}

// The sums of two parts.  (A part of -infinities alone has a sum of 0, or NaN.)
__device__ __forceinline__ Part joined(const Distill& D, Part a, Part b) {
    const float top = fmaxf(a.top, b.top), to = top == -INFINITY ? 0.f : top;
    return {top, a.sum * exp2_of((a.top - to) * D.to_log2) + b.sum * exp2_of((b.top - to) * D.to_log2)};
}

struct Max {
    static __device__ __forceinline__ float of(float a, float b) { return fmaxf(a, b); }
};
struct Sum {
    static __device__ __forceinline__ float of(float a, float b) { return a + b; }
};

// N values over LANES adjacent threads each.  Of more than a wave, `room` has N places for each wave.
template <typename Op, int LANES, int N>
__device__ __forceinline__ void over_lanes(float (&v)[N], float* room) {
#pragma unroll
    for (int d = (LANES < 64 ? LANES : 64) / 2; d; d >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = Op::of(v[n], __shfl_xor(v[n], d));
    if constexpr (LANES > 64) {
        __syncthreads();                 // (the room may still be read)
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int n = 0; n < N; ++n) room[(threadIdx.x >> 6) * N + n] = v[n];
        __syncthreads();
#pragma unroll
        for (int n = 0; n < N; ++n) v[n] = room[n];
#pragma unroll
        for (int w = 1; w < LANES / 64; ++w)
#pragma unroll
            for (int n = 0; n < N; ++n) v[n] = Op::of(v[n], room[w * N + n]);
    }
}

// 4 W bytes of adjacent logits, as words: their values unpack where they are used.
template <typename T, int W = 4>
struct Logits {
    static constexpr int E = 4 * W / (int)sizeof(T);
    uint32_t w[W];

    __device__ __forceinline__ float value(int e) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
        else return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    }
    // None: -infinity.
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    }
    // PAST: around the caches.
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T* p) {
        using Words = __attribute__((ext_vector_type(W), aligned(sizeof(T)))) uint32_t;
        const Words* const q = reinterpret_cast<const Words*>(p);
        const Words v = PAST ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int i = 0; i < W; ++i) w[i] = v[i];
    }
    // Those from p on, -infinity for those from n on.
    template <bool PAST = false>
    __device__ __forceinline__ void load(const T* p, int64_t n) {
        clear();
        if (n >= E) {
            load<PAST>(p);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < n) {
                    if constexpr (sizeof(T) == 4) w[e] = __builtin_bit_cast(uint32_t, p[e]);
                    else w[e / 2] = e & 1 ? (w[e / 2] & 0xffffu) | (uint32_t)p[e] << 16 : (w[e / 2] & 0xffff0000u) | p[e];
                }
        }
    }
    __device__ __forceinline__ float top(float of) const {
#pragma unroll
        for (int e = 0; e < E; ++e) of = fmaxf(of, value(e));
        return of;
    }
    // The same words, of which the compiler knows no more: bfloat16 unpacked for one pass is not kept
    // for the next one, for which there are no registers.
    __device__ __forceinline__ void forget() {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < W; ++i) asm volatile("" : "+v"(w[i]));
        }
    }
};

// E gradients from p on, the first n of them.
template <bool PAST, typename T, int E>
__device__ __forceinline__ void store_gradients(T* p, const float (&v)[E], int64_t n) {
    if (n >= E) {
        using Words = __attribute__((ext_vector_type(E * sizeof(T) / 4), aligned(sizeof(T)))) uint32_t;
        Words w;
#pragma unroll
        for (int i = 0; i < (int)(E * sizeof(T) / 4); ++i) {
            if constexpr (sizeof(T) == 4) {
                w[i] = __float_as_uint(v[i]);
            } else {                     // (two at a time: one instruction)
                using f32x2 = __attribute__((ext_vector_type(2))) float;
                using bf16x2 = __attribute__((ext_vector_type(2))) __bf16;
                w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
            }
        }
        if constexpr (PAST) __builtin_nontemporal_store(w, reinterpret_cast<Words*>(p));
        else *reinterpret_cast<Words*>(p) = w;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < n) store_elem(p + e, v[e]);
    }
}

}  // namespace dss
