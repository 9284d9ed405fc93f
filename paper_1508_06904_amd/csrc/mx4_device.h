// Device helpers of the 4-bit tokens: a block's scale, its codes, and a layer's outputs.
#pragma once

#include "mx4.h"
#include "tokens_device.h"

namespace dss {

using f32x4 = __attribute__((ext_vector_type(4))) float;

// The scale byte of a block from its largest |x|'s bits: the exponent less 2, so that the largest
// value comes to lie in [4, 8); 255 (NaN) if that is no finite number.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    return top >= kInfBits ? 255u : (uint32_t)max((int)(top >> 23) - 2, 0);
}

// 2^(byte - 127) as the conversions take it: they read the exponent's bits alone, those of 2^-127 (0) too.
__device__ __forceinline__ float scale_operand(uint32_t byte) { return __uint_as_float(byte << 23); }

// Eight codes of adjacent channels: v_cvt_scalef32_pk_fp4_f32 divides by the scale and rounds to the
// nearest code, ties to the even one, and to 6 from above it; signs are kept.
__device__ __forceinline__ uint32_t eight_codes(const float (&v)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

// Eight adjacent channels of a row, a quarter of a block: four adjacent lanes have a block.
template <typename T>
struct Eight {
    Chunk<T> c[8 / Chunk<T>::E];

    // From p on, those from n on as zeros (n may be negative).
    __device__ __forceinline__ void load(const T* p, int64_t n) {
#pragma unroll
        for (int i = 0; i < 8 / Chunk<T>::E; ++i)
            c[i] = load_chunk(p + i * Chunk<T>::E, (int)max(min(n - i * Chunk<T>::E, (int64_t)8), (int64_t)0));
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < 8 / Chunk<T>::E; ++i) c[i] = Chunk<T>{};
    }
    // The scale of the four lanes' block.
    __device__ __forceinline__ uint32_t scale_byte_of_four() const {
        uint32_t t = 0;
#pragma unroll
        for (int i = 0; i < 8 / Chunk<T>::E; ++i) t = raise(t, c[i]);
        t = top_bits<T>(t);
        t = max(t, (uint32_t)__shfl_xor((int)t, 1));
        t = max(t, (uint32_t)__shfl_xor((int)t, 2));
        return scale_byte(t);
    }
    __device__ __forceinline__ uint32_t codes(uint32_t byte) const {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c[k / Chunk<T>::E].value(k % Chunk<T>::E);
        return byte == 255u ? 0u : eight_codes(v, scale_operand(byte));
    }
};

// A block of n channels from p on, `stride` apart: its codes, and its scale in `byte`.
template <typename T>
__device__ __forceinline__ i32x4 block_codes(const T* p, int64_t stride, int n, uint32_t& byte) {
    float v[kBlock];
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kBlock; ++k) {
        v[k] = k < n ? to_f32(p[k * stride]) : 0.f;
        top = max(top, abs_bits(v[k]));
    }
    byte = scale_byte(top);
    i32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float e[8] = {v[8 * j], v[8 * j + 1], v[8 * j + 2], v[8 * j + 3], v[8 * j + 4], v[8 * j + 5], v[8 * j + 6], v[8 * j + 7]};
        w[j] = byte == 255u ? 0 : (int)eight_codes(e, scale_operand(byte));
    }
    return w;
}

// A block of 32 channels of V adjacent tokens of a map (W words of each channel), which a lane has in registers.
template <typename T, int W = 4>
struct MapBlock {
    static constexpr int V = 4 * W / (int)sizeof(T);
    static constexpr int kTokens = 16 * V;             // of a wave, of whose lanes 16 have adjacent tokens
    uint32_t w[kBlock][W];

    // Channel k of the block, token j.
    __device__ __forceinline__ float value(int k, int j) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[k][j]);
        else return __uint_as_float(j & 1 ? w[k][j / 2] & 0xffff0000u : w[k][j / 2] << 16);
    }
    __device__ __forceinline__ void load(const T* p, int64_t ks, int n) {
#pragma unroll
        for (int k = 0; k < kBlock; ++k) {
#pragma unroll
            for (int i = 0; i < W; ++i) w[k][i] = 0;
            if (k < n) __builtin_memcpy(w[k], p + k * ks, 4 * W);
        }
    }
    __device__ __forceinline__ void scale_bytes(uint32_t (&byte)[V]) const {
        uint32_t top[W] = {};
#pragma unroll
        for (int k = 0; k < kBlock; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i) top[i] = raise<T>(top[i], w[k][i]);
#pragma unroll
        for (int j = 0; j < V; ++j)
            byte[j] = scale_byte(sizeof(T) == 4 ? top[j] : j & 1 ? top[j / 2] & 0xffff0000u : top[j / 2] << 16);
    }
    // The 32 codes of token j.
    __device__ __forceinline__ i32x4 codes(int j, uint32_t byte) const {
        const float scale = scale_operand(byte);
        i32x4 r;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = value(8 * q + k, j);
            r[q] = (int)(byte == 255u ? 0u : eight_codes(v, scale));
        }
        return r;
    }
};

// c + the product of 16 rows of 128 codes each with 16 others. A lane has 32 adjacent codes of row
// (lane & 15), block (lane >> 4), and their scale in the lowest byte of a_scale and in BYTE of b_scale; row r of the first operand and row
// l of the second meet in lane (l, r >> 2), register r & 3.
template <int BYTE>
__device__ __forceinline__ f32x4 multiply_byte(i32x4 a, uint32_t a_scale, i32x4 b, uint32_t b_scale, f32x4 c) {
    using i32x8 = __attribute__((ext_vector_type(8))) int;
    const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const i32x8 b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, (int)a_scale, BYTE, (int)b_scale);
}
// (A byte that is constant once the loops are unrolled.)
__device__ __forceinline__ f32x4 multiply_at(int byte, i32x4 a, uint32_t a_scale, i32x4 b, uint32_t b_scale, f32x4 c) {
    switch (byte & 3) {
        case 0: return multiply_byte<0>(a, a_scale, b, b_scale, c);
        case 1: return multiply_byte<1>(a, a_scale, b, b_scale, c);
        case 2: return multiply_byte<2>(a, a_scale, b, b_scale, c);
        default: return multiply_byte<3>(a, a_scale, b, b_scale, c);
    }
}

// The activation of N outputs, chosen once: a branch for each of them cost a 4-bit layer on a map half of its time.
template <int N>
__device__ __forceinline__ void activate_all(int act, float (&v)[N]) {
    if (act == DSS_ACT_RELU) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = activate_nan(DSS_ACT_RELU, v[k]);
    } else if (act == DSS_ACT_TANH) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = activate_nan(DSS_ACT_TANH, v[k]);
    }
}

// N adjacent outputs from p on, which has place j of J; those past the end are left out.
template <typename Tout, int N>
__device__ __forceinline__ void store_values(Tout* p, const float (&v)[N], int64_t j, int64_t J, int past) {
    constexpr int C = N * (int)sizeof(Tout) < 16 ? N : 16 / (int)sizeof(Tout);   // outputs of one store
#pragma unroll
    for (int c = 0; c < N; c += C) {
        struct {
            Tout v[C];
        } r;
#pragma unroll
        for (int k = 0; k < C; ++k) store_elem(&r.v[k], v[c + k]);
        if (j + c + C <= J) {
            using Words = __attribute__((ext_vector_type(C * sizeof(Tout) / 4), aligned(sizeof(Tout)))) uint32_t;
            if (past) __builtin_nontemporal_store(__builtin_bit_cast(Words, r), reinterpret_cast<Words*>(p + c));
            else __builtin_memcpy(p + c, &r, sizeof r);
        } else {
#pragma unroll
            for (int k = 0; k < C; ++k)
                if (j + c + k < J) p[c + k] = r.v[k];
        }
    }
}

}  // namespace dss
