// Device helpers of the 8-bit tokens: a token's scale and its codes.
//
// The largest absolute value of a token is taken over the bit patterns: without
// their sign bits these order as the values do, and infinities and NaN come out
// above all finite ones, which a floating maximum would lose.
#pragma once

#include "dev_common.h"

namespace dss {

constexpr uint32_t kInfBits = 0x7f800000u;

template <typename T>
struct Chunk {                            // 16 bytes of a row
    static constexpr int E = 16 / (int)sizeof(T);
    T v[E];
};

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The scale of a token from its largest |x|'s bits: NaN if that is no number.
__device__ __forceinline__ float scale_of(uint32_t bits) {
    return bits >= kInfBits ? __uint_as_float(0x7fc00000u) : __uint_as_float(bits) / 127.f;
}

// One code.  A scale of 0 or NaN gives 0 for every value (the quotient could be anything).
__device__ __forceinline__ int code_of(float v, float scale) {
    const float q = fminf(fmaxf(rintf(v / scale), -127.f), 127.f);
    return scale > 0.f ? (int)q : 0;
}

// E consecutive values from p on, those from n on as zeros (n may be negative).
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
    Chunk<T> r;
    if (n >= Chunk<T>::E) {
        __builtin_memcpy(&r, p, 16);
    } else {
#pragma unroll
        for (int k = 0; k < Chunk<T>::E; ++k) r.v[k] = k < n ? p[k] : T(0);
    }
    return r;
}

// The E codes of a chunk to p, those from n on left out.
template <typename T>
__device__ __forceinline__ void store_codes(int8_t* p, const Chunk<T>& x, float scale, int n) {
    constexpr int E = Chunk<T>::E;
    uint32_t w[E / 4];
#pragma unroll
    for (int j = 0; j < E / 4; ++j) {
        w[j] = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) w[j] |= (uint32_t)(code_of(to_f32(x.v[4 * j + k]), scale) & 0xff) << (8 * k);
    }
    if (n >= E) {
        __builtin_memcpy(p, w, E);
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) p[k] = (int8_t)(w[k / 4] >> (8 * (k % 4)));
    }
}

}  // namespace dss
