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

// Codes of one token: rint(x / scale) of the binary32 quotient, clamped, as the low byte.
//
// The quotient is the correctly rounded one without a division for each value:
// with r the nearest number to 1 / scale, two steps q += (x - q scale) r from
// q = x r end at the number nearest to x / scale, since the first one leaves q
// within its last place of the quotient (P. Markstein, Computation of elementary
// functions on the IBM RISC System/6000 processor, 1990).  The remainders are exact
// while they stay above the smallest numbers: below a scale of 2^-100 the division
// is made after all (there a quotient may also need the clamping: of a normal
// scale no |x| <= 127 scale is over 127 by more than its rounding).  Adding
// 1.5 * 2^23 rounds to an integer, ties to even, whose low byte is the code.
struct Coder {
    float scale, r;
    uint32_t keep;                        // no bits where the scale is 0 or NaN: those codes are 0
    bool tiny;

    __device__ __forceinline__ explicit Coder(float s) : scale(s), r(1.f / s), keep(s > 0.f ? ~0u : 0u), tiny(s < 0x1p-100f) {}

    __device__ __forceinline__ uint32_t bits(float x) const {
        float q = x * r;
        q = fmaf(fmaf(-q, scale, x), r, q);
        q = fmaf(fmaf(-q, scale, x), r, q);
        return __float_as_uint(q + 0x1.8p23f);
    }
    __device__ __forceinline__ uint32_t tiny_bits(float x) const {
        return __float_as_uint(fminf(fmaxf(x / scale, -127.f), 127.f) + 0x1.8p23f);
    }
    // Four codes of adjacent channels.
    __device__ __forceinline__ uint32_t four(float a, float b, float c, float d) const {
        const uint32_t w[4] = {tiny ? tiny_bits(a) : bits(a), tiny ? tiny_bits(b) : bits(b), tiny ? tiny_bits(c) : bits(c),
                               tiny ? tiny_bits(d) : bits(d)};
        const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
        return (lo | hi) & keep;
    }
    __device__ __forceinline__ int8_t one(float x) const { return (int8_t)((tiny ? tiny_bits(x) : bits(x)) & keep); }
};

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

// A lane's chunks of a row of K values: chunk i starts at (i * lanes + lane) * E; zeros from K on.
// All whole chunks first, so that their loads are under way together.
template <typename T, int CH>
__device__ __forceinline__ void load_row(Chunk<T> (&c)[CH], const T* row, int lane, int lanes, int K) {
    constexpr int E = Chunk<T>::E;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int at = (i * lanes + lane) * E;
        c[i] = Chunk<T>{};
        if (at + E <= K) __builtin_memcpy(&c[i], row + at, 16);
    }
    if (K % E == 0) return;
    const int last = K / E;              // the chunk that K ends in
#pragma unroll
    for (int i = 0; i < CH; ++i)
        if (i * lanes + lane == last) {
#pragma unroll
            for (int k = 0; k < E - 1; ++k)
                if (last * E + k < K) c[i].v[k] = row[last * E + k];
        }
}

// The E codes of a chunk to p, those from n on left out.
template <typename T>
__device__ __forceinline__ void store_codes(int8_t* p, const Chunk<T>& x, const Coder& coder, int n) {
    constexpr int E = Chunk<T>::E;
    uint32_t w[E / 4];
#pragma unroll
    for (int j = 0; j < E / 4; ++j)
        w[j] = coder.four(to_f32(x.v[4 * j]), to_f32(x.v[4 * j + 1]), to_f32(x.v[4 * j + 2]), to_f32(x.v[4 * j + 3]));
    if (n >= E) {
        __builtin_memcpy(p, w, E);
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) p[k] = (int8_t)(w[k / 4] >> (8 * (k % 4)));
    }
}

}  // namespace dss
