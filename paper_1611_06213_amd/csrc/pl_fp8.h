// Conversion of fp32 and bf16 to 8-bit floating point with a power-of-two scale per block:
//
// e = the least whole number >= -126 with max|x| <= 448 * 2^e over a block's finite elements;
// element = x * 2^-e rounded to nearest even e4m3. 448 = 1.75 * 2^8, so e comes from the bits of
// the maximum: its exponent field once the mantissa is rounded up past 1.75, less 8.
#pragma once

#include "pl_device.h"

namespace gadei::learner {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef int16_t i16x2 __attribute__((ext_vector_type(2)));

// The scale's byte (exponent + 127) for the largest finite |x| of a block, as its bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
    const uint32_t e = (bits + 0x1fffffu) >> 23;
    return e < 9 ? 1 : e - 8;
}

// Magnitudes compare as their bits do. Those of bf16 are compared two at a time, as loaded.
template <int X> struct Mags;

template <> struct Mags<PS_F32> {
    static constexpr int kWords = 8;   // of eight elements
    static constexpr uint32_t kInf = 0x7f800000u;
    static __device__ __forceinline__ uint32_t word(const Bits8<PS_F32> &r, int i) {
        return __float_as_uint(i < 4 ? r.a[i] : r.b[i - 4]) & 0x7fffffffu;
    }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) { return max(a, b); }
    static __device__ __forceinline__ uint32_t finite(uint32_t a) { return a < kInf ? a : 0; }
    // of the words' elements, as fp32 bits
    static __device__ __forceinline__ uint32_t element(const uint32_t (&w)[8], int e) { return w[e]; }
    static __device__ __forceinline__ uint32_t of_all(uint32_t w) { return w; }
};

template <> struct Mags<PS_BF16> {
    static constexpr int kWords = 4;
    static constexpr uint32_t kInf = 0x7f800000u;
    static __device__ __forceinline__ uint32_t word(const Bits8<PS_BF16> &r, int i) { return r.a[i] & 0x7fff7fffu; }
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                      __builtin_bit_cast(u16x2, b)));
    }
    static __device__ __forceinline__ uint32_t finite(uint32_t a) {
        const uint32_t lo = (a & 0xffffu) < 0x7f80u ? a & 0xffffu : 0, hi = a < kInf ? a & 0xffff0000u : 0;
        return lo | hi;
    }
    static __device__ __forceinline__ uint32_t element(const uint32_t (&w)[4], int e) {
        return e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16;
    }
    static __device__ __forceinline__ uint32_t of_all(uint32_t w) { return max(w << 16, w & 0xffff0000u); }
};

// Two elements of a row, or of neighbouring rows, x * 2^(127 - byte) in e4m3, into the lower or
// upper half of a word. One instruction converts and scales: by a power of two, so that it rounds
// once. NaN and infinities become NaN (e4m3 has no infinity).
template <bool UPPER>
__device__ __forceinline__ uint32_t pair_f32(uint32_t into, float a, float b, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(
                                            __builtin_bit_cast(i16x2, into), a, b, scale, UPPER));
}
template <bool UPPER>
__device__ __forceinline__ uint32_t pair_bf16(uint32_t into, uint32_t ab, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
                                            __builtin_bit_cast(i16x2, into), __builtin_bit_cast(bf16x2, ab), scale, UPPER));
}

// Four neighbours of a row, the first (h = 0) or last of its eight.
__device__ __forceinline__ uint32_t four(const Bits8<PS_F32> &r, int h, float scale) {
    const f32x4 v = h == 0 ? r.a : r.b;
    return pair_f32<true>(pair_f32<false>(0, v[0], v[1], scale), v[2], v[3], scale);
}
__device__ __forceinline__ uint32_t four(const Bits8<PS_BF16> &r, int h, float scale) {
    return pair_bf16<true>(pair_bf16<false>(0, r.a[2 * h], scale), r.a[2 * h + 1], scale);
}

// Element e of four neighbouring rows.
__device__ __forceinline__ uint32_t four_rows(const Bits8<PS_F32> *r, int e, float scale) {
    auto at = [&](int i) { return e < 4 ? r[i].a[e] : r[i].b[e - 4]; };
    return pair_f32<true>(pair_f32<false>(0, at(0), at(1), scale), at(2), at(3), scale);
}
__device__ __forceinline__ uint32_t four_rows(const Bits8<PS_BF16> *r, int e, float scale) {
    auto two = [&](int i) {   // of rows i and i + 1
        const uint32_t a = r[i].a[e >> 1], b = r[i + 1].a[e >> 1];
        return e & 1 ? __builtin_amdgcn_perm(b, a, 0x07060302) : __builtin_amdgcn_perm(b, a, 0x05040100);
    };
    return pair_bf16<true>(pair_bf16<false>(0, two(0), scale), two(2), scale);
}

__device__ __forceinline__ float as_scale(uint32_t byte) { return __uint_as_float(byte << 23); }


// The largest finite magnitude of a lane's eight elements, as fp32 bits.
template <int X>
__device__ __forceinline__ uint32_t most8(const Bits8<X> &x) {
    using M = Mags<X>;
    uint32_t m = 0;
#pragma unroll
    for (int w = 0; w < M::kWords; ++w) m = M::most(m, M::word(x, w));
    if (M::of_all(m) >= M::kInf) {   // rare: without what is not finite
        m = 0;
#pragma unroll
        for (int w = 0; w < M::kWords; ++w) m = M::most(m, M::finite(M::word(x, w)));
    }
    return M::of_all(m);
}

// Of the block's 128, which sixteen neighbouring lanes hold.
__device__ __forceinline__ uint32_t most_of_block(uint32_t m) {
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(m, d)));
    return m;
}

}  // namespace gadei::learner
