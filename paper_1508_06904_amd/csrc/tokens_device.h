// Device helpers of the 8-bit tokens: a token's scale and its codes, and a layer's
// outputs from the sums of products.
//
// The largest absolute value of a token is taken over the bit patterns: without
// their sign bits these order as the values do, and infinities and NaN come out
// above all finite ones, which a floating maximum would lose.
#pragma once

#include "dev_common.h"
#include "tokens.h"

namespace dss {

constexpr uint32_t kInfBits = 0x7f800000u;

// Workgroups are handed to the 8 XCDs in turn: the id of the tile that makes the
// tiles of one XCD (and of its L2) neighbours.
__device__ __forceinline__ int64_t xcd_order(int64_t b, int64_t n) {
    const int64_t x = b & 7, q = n >> 3, r = n & 7;
    return x * q + min(x, r) + (b >> 3);
}

// 16 bytes of a row, as words: their values unpack where they are used.
template <typename T>
struct Chunk {
    static constexpr int E = 16 / (int)sizeof(T);
    uint32_t w[4] = {};

    __device__ __forceinline__ float value(int k) const {
        if constexpr (E == 4) return __uint_as_float(w[k]);
        else return __uint_as_float(k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16);
    }
    __device__ __forceinline__ void set(int k, T v) {  // (over a zero)
        if constexpr (E == 4) w[k] = __builtin_bit_cast(uint32_t, v);
        else w[k / 2] |= (uint32_t)v << (16 * (k & 1));
    }
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

// The largest |value| so far of each of a word's values: of one, or of two at a time.
template <typename T>
__device__ __forceinline__ uint32_t raise(uint32_t top, uint32_t word) {
    if constexpr (sizeof(T) == 4) {
        return max(top, word & 0x7fffffffu);
    } else {
        using u16x2 = __attribute__((ext_vector_type(2))) uint16_t;
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, top),
                                                                      __builtin_bit_cast(u16x2, word & 0x7fff7fffu)));
    }
}
template <typename T>
__device__ __forceinline__ uint32_t raise(uint32_t top, const Chunk<T>& c) {
#pragma unroll
    for (int k = 0; k < 4; ++k) top = raise<T>(top, c.w[k]);
    return top;
}
// The bits of the largest of a word's values, as binary32.
template <typename T>
__device__ __forceinline__ uint32_t top_bits(uint32_t top) {
    return sizeof(T) == 4 ? top : max(top << 16, top & 0xffff0000u);
}

// E consecutive values from p on, those from n on as zeros (n may be negative).
template <typename T>
__device__ __forceinline__ Chunk<T> load_chunk(const T* p, int n) {
    Chunk<T> r;
    if (n >= Chunk<T>::E) {
        __builtin_memcpy(&r, p, 16);
    } else {
#pragma unroll
        for (int k = 0; k < Chunk<T>::E; ++k)
            if (k < n) r.set(k, p[k]);
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
                if (last * E + k < K) c[i].set(k, row[last * E + k]);
        }
}

// The E codes of a chunk to p, those from n on left out.
template <typename T>
__device__ __forceinline__ void store_codes(int8_t* p, const Chunk<T>& x, const Coder& coder, int n) {
    constexpr int E = Chunk<T>::E;
    uint32_t w[E / 4];
#pragma unroll
    for (int j = 0; j < E / 4; ++j)
        w[j] = coder.four(x.value(4 * j), x.value(4 * j + 1), x.value(4 * j + 2), x.value(4 * j + 3));
    if (n >= E) {
        __builtin_memcpy(p, w, E);
    } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
            if (k < n) p[k] = (int8_t)(w[k / 4] >> (8 * (k % 4)));
    }
}

// ------------------------------------------------------------------ tiles of a map
// A workgroup of up to kMapWaves waves holds kLaneTokens * 16 adjacent tokens of up to
// 64 channels for each wave in registers.  16 lanes read 16 bytes each of one channel, 256 adjacent
// bytes; a lane keeps 16 adjacent channels of its tokens, so that each token's
// codes leave it as 16 bytes, with no turning round through LDS.
constexpr int kMapWaves = 16;

template <typename T>
struct MapTile {
    static constexpr int V = 16 / (int)sizeof(T);      // tokens of a lane
    static constexpr int kTokens = 16 * V;
    Chunk<T> c[16];                                    // c[r].value(j): channel r of the lane's group, token j

    // The tile's tokens start at x; the lane's channels k .. k+15, those below K.
    __device__ __forceinline__ void load(const T* x, int64_t channel_stride, uint32_t k, uint32_t K) {
        const T* p = x + (threadIdx.x & 15) * V + k * channel_stride;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            c[r] = Chunk<T>{};
            if (k + r < K) __builtin_memcpy(&c[r], p + r * channel_stride, 16);
        }
    }
    __device__ __forceinline__ void raise_into(uint32_t (&top)[4]) const {
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) top[j] = raise<T>(top[j], c[r].w[j]);
    }
    // Each of the lane's tokens' largest value over the lanes of the `waves` waves from `first`
    // on, which share a tile; tops has 64 words for each wave of the workgroup.
    static __device__ __forceinline__ void meet(uint32_t (&top)[4], uint32_t* tops, int first, int waves) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            top[j] = raise<T>(top[j], (uint32_t)__shfl_xor((int)top[j], 16));
            top[j] = raise<T>(top[j], (uint32_t)__shfl_xor((int)top[j], 32));
        }
        if (lane < 16)
#pragma unroll
            for (int j = 0; j < 4; ++j) tops[((threadIdx.x >> 6) * 16 + lane) * 4 + j] = top[j];
        __syncthreads();
        for (int w = first; w < first + waves; ++w)
#pragma unroll
            for (int j = 0; j < 4; ++j) top[j] = raise<T>(top[j], tops[(w * 16 + (lane & 15)) * 4 + j]);
    }
    // Token j's of these.
    static __device__ __forceinline__ uint32_t bits(const uint32_t (&top)[4], int j) {
        if constexpr (V == 4) return top[j];
        else return j & 1 ? top[j / 2] & 0xffff0000u : top[j / 2] << 16;
    }
    // The 16 codes of token j's channels.
    __device__ __forceinline__ void codes(int j, const Coder& coder, uint32_t (&w)[4]) const {
#pragma unroll
        for (int q = 0; q < 4; ++q)
            w[q] = coder.four(c[4 * q].value(j), c[4 * q + 1].value(j), c[4 * q + 2].value(j), c[4 * q + 3].value(j));
    }
};

// ------------------------------------------------------------------ outputs of a layer
using i32x4 = __attribute__((ext_vector_type(4))) int;

// A NaN stays one (fmaxf would make it 0).
__device__ __forceinline__ float activate_nan(int act, float v) {
    if (act == DSS_ACT_RELU) return v < 0.f ? 0.f : v;
    if (act == DSS_ACT_TANH) return tanhf(v);
    return v;
}

__device__ __forceinline__ float output_of(int sum, float wscale, float scale, float bias, int act) {
    return activate_nan(act, (float)sum * wscale * scale + bias);
}

// What a lane's outputs need besides their sums: D's side i (one value) and side j
// (N adjacent ones).  Read before the first output is stored: to the compiler a
// store may change any of it.
struct Side1 {
    float scale, bias;
};
template <int N>
struct SideN {
    float scale[N], bias[N];
};
template <bool MAP>
__device__ __forceinline__ Side1 side_i(const Layer& L, int64_t i) {
    if constexpr (MAP) {
        i = min(i, (int64_t)L.N - 1);
        return {L.weight_scales[i], L.bias ? L.bias[i] : 0.f};
    } else {
        return {L.scales[min(i, L.M - 1)], 0.f};
    }
}
template <bool MAP, int N = 4>
__device__ __forceinline__ SideN<N> side_j(const Layer& L, int64_t j) {
    SideN<N> r;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t at = min(j + k, MAP ? L.M - 1 : (int64_t)L.N - 1);
        r.scale[k] = MAP ? L.scales[at] : L.weight_scales[at];
        r.bias[k] = !MAP && L.bias ? L.bias[at] : 0.f;
    }
    return r;
}

// N adjacent outputs D[i][j .. j+N-1] of a layer, those before j_first and from J on left out; sum[N / 4].
template <typename Tout, bool MAP, int N>
__device__ __forceinline__ void store_outputs(const Layer& L, int64_t i, int64_t j, int64_t J, const i32x4* sum,
                                              const Side1& P, const SideN<N>& Q, int64_t j_first = 0) {
    constexpr int C = N * (int)sizeof(Tout) < 16 ? N : 16 / (int)sizeof(Tout);   // outputs of one store
    Tout* p = static_cast<Tout*>(L.out) + i * L.ldo + j;
#pragma unroll
    for (int c = 0; c < N; c += C) {
        struct {
            Tout v[C];
        } r;
#pragma unroll
        for (int k = 0; k < C; ++k) {
            const int s = sum[(c + k) / 4][(c + k) % 4];
            store_elem(&r.v[k], MAP ? output_of(s, P.scale, Q.scale[c + k], P.bias, L.act)
                                    : output_of(s, Q.scale[c + k], P.scale, Q.bias[c + k], L.act));
        }
        if (j + c >= j_first && j + c + C <= J) {
            if constexpr (sizeof(Tout) * C == 16) {
                using u32x4 = __attribute__((ext_vector_type(4), aligned(sizeof(Tout)))) uint32_t;
                if (L.past) __builtin_nontemporal_store(__builtin_bit_cast(u32x4, r), reinterpret_cast<u32x4*>(p + c));
                else __builtin_memcpy(p + c, &r, sizeof r);
            } else {
                __builtin_memcpy(p + c, &r, sizeof r);
            }
        } else {
#pragma unroll
            for (int k = 0; k < C; ++k)
                if (j + c + k >= j_first && j + c + k < J) p[c + k] = r.v[k];
        }
    }
}

// 16 bytes from any address, out of five aligned words: a 16-byte load that starts inside a word
// takes several times as long.  Where one of the words would leave [begin, end) the load is that one.
__device__ __forceinline__ i32x4 load_any(const int8_t* p, const int8_t* begin, const int8_t* end) {
    i32x4 v;
    const int shift = (int)((uintptr_t)p & 3);
    const int8_t* q = p - shift;
    if (q < begin || q + 20 > end) {
        __builtin_memcpy(&v, p, 16);
        return v;
    }
    using words = __attribute__((ext_vector_type(4), aligned(4))) int;
    const words w = *reinterpret_cast<const words*>(q);
    const int last = *reinterpret_cast<const int*>(q + 16);
    v[0] = __builtin_amdgcn_alignbyte(w[1], w[0], shift);
    v[1] = __builtin_amdgcn_alignbyte(w[2], w[1], shift);
    v[2] = __builtin_amdgcn_alignbyte(w[3], w[2], shift);
    v[3] = __builtin_amdgcn_alignbyte(last, w[3], shift);
    return v;
}

// Bytes k .. k+15 of a row of K bytes, zeros past its end; nothing past the end is read.
__device__ __forceinline__ i32x4 load_unit(const int8_t* row, int k, int K) {
    i32x4 v = {};
    if (k + 16 <= K) {
        __builtin_memcpy(&v, row + k, 16);
    } else if (k < K) {
        if (K >= 16) {
            unsigned __int128 w;
            __builtin_memcpy(&w, row + K - 16, 16);
            w >>= 8 * (k + 16 - K);
            __builtin_memcpy(&v, &w, 16);
        } else {
            for (int b = 0; b < K - k; ++b) v[b >> 2] |= (int)(uint8_t)row[k + b] << (8 * (b & 3));
        }
    }
    return v;
}

}  // namespace dss
