// Matrices to 8-bit floating point with a power-of-two scale per block of 128.
//
// Mathematics: e = the least whole number >= -126 with max|x| <= 448 * 2^e over a block's
// finite elements; element = x * 2^-e rounded to nearest even e4m3. 448 = 1.75 * 2^8, so
// e comes from the bits of the maximum: its exponent field once the mantissa is
// rounded up past 1.75, less 8.
//
// Bound by memory: x is read once and one byte per element written for each layout. A
// workgroup takes a 128 x 128 tile of x: sixteen lanes hold a row's 128 elements, eight
// each, so a row's maximum is a reduction over sixteen lanes; columns' maxima and the
// transposed bytes go through LDS.
#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kBlock = 256;
constexpr int kTile = 128;
constexpr int kRows = 8;   // a thread's rows: four neighbours, and the four 64 rows on

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

// Where word w (four rows) of column c of the transposed tile lies: fours of words exchanged by
// the column, so that neither the writes (16 columns eight apart, four words of each) nor
// the reads (four words of a column together) meet in a bank.
__device__ __forceinline__ int word_at(int c, int w) {
    return 32 * (c ^ ((c >> 6) & 1)) + (w ^ (((c >> 3) & 7) << 2));
}

template <int X, bool SQUARE>
__global__ __launch_bounds__(kBlock) void quantize_tile(QuantArgs a, uint32_t tiles_x) {
    using M = Mags<X>;
    constexpr int W = M::kWords;
    __shared__ uint32_t col_max[kTile];
    __shared__ __attribute__((aligned(16))) uint32_t columns[kTile * 32];
    __shared__ uint32_t all_max;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x / tiles_x) * kTile;
    const int64_t tile_x = blockIdx.x % tiles_x, c0 = tile_x * kTile;
    const int g = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t col = c0 + 8 * g;
    const int count = a.cols - col >= 8 ? 8 : a.cols > col ? static_cast<int>(a.cols - col) : 0;
    const bool transposed = a.values_t != nullptr;
    if (threadIdx.x < kTile) col_max[threadIdx.x] = 0;
    if (threadIdx.x == 0) all_max = 0;

    auto row_of = [&](int i) { return r0 + 4 * y + (i & 3) + 64 * (i >> 2); };
    Bits8<X> x[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const int64_t r = row_of(i);
        if (r < a.rows && count == 8) x[i] = load8<X>(a.x, r * a.ld + col);
        else x[i] = load8_some<X>(a.x, r * a.ld + col, r < a.rows ? count : 0);
    }
    uint32_t row_max[kRows];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int w = 0; w < W; ++w) m = M::most(m, M::word(x[i], w));
        if (M::of_all(m) >= M::kInf) {   // rare: without what is not finite
            m = 0;
#pragma unroll
            for (int w = 0; w < W; ++w) m = M::most(m, M::finite(M::word(x[i], w)));
        }
        m = M::of_all(m);
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(m, d)));
        row_max[i] = m;
        most = max(most, m);
    }
    if constexpr (SQUARE) {
        __syncthreads();
        if (g == 0) atomicMax(&all_max, most);
        __syncthreads();
        most = all_max;
#pragma unroll
        for (int i = 0; i < kRows; ++i) row_max[i] = most;
    }
    if (a.values != nullptr) {
        const int64_t ld = (a.cols + 127) / 128 * 128;
        const int64_t words = (tile_x >> 2) * a.rows;   // of scales before this group's
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t r = row_of(i);
            if (r >= a.rows) continue;
            const uint32_t byte = scale_byte(row_max[i]);
            *reinterpret_cast<u32x2 *>(a.values + r * ld + col) =
                u32x2{four(x[i], 0, as_scale(byte)), four(x[i], 1, as_scale(byte))};
            if (g == 0)
                reinterpret_cast<uint8_t *>(a.scales + words + r)[tile_x & 3] = static_cast<uint8_t>(byte);
        }
    }
    if (!transposed) return;

    uint32_t col_byte[8];
    if constexpr (SQUARE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) col_byte[e] = scale_byte(most);
    } else {
        __syncthreads();
        uint32_t m[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            m[w] = 0;
#pragma unroll
            for (int i = 0; i < kRows; ++i) m[w] = M::most(m[w], M::word(x[i], w));
            if (M::of_all(m[w]) >= M::kInf) {
                m[w] = 0;
#pragma unroll
                for (int i = 0; i < kRows; ++i) m[w] = M::most(m[w], M::finite(M::word(x[i], w)));
            }
            // the wave's four rows of lanes
            m[w] = M::most(m[w], static_cast<uint32_t>(__shfl_xor(m[w], 16)));
            m[w] = M::most(m[w], static_cast<uint32_t>(__shfl_xor(m[w], 32)));
        }
        if ((threadIdx.x & 63) < 16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) atomicMax(&col_max[8 * g + e], M::element(m, e));
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) col_byte[e] = scale_byte(col_max[8 * g + e]);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int h = 0; h < kRows / 4; ++h)
            columns[word_at(8 * g + e, y + 16 * h)] = four_rows(x + 4 * h, e, as_scale(col_byte[e]));
    __syncthreads();
    const int64_t ld_t = (a.rows + 127) / 128 * 128;
    // 128 columns of x, 128 bytes each: eight lanes a column
#pragma unroll
    for (int i = threadIdx.x; i < kTile * 8; i += kBlock) {
        const int c = i >> 3, w = 4 * (i & 7);
        if (c0 + c < a.cols)
            *reinterpret_cast<u32x4 *>(a.values_t + (c0 + c) * ld_t + r0 + 4 * w) =
                *reinterpret_cast<const u32x4 *>(columns + word_at(c, w));
    }
    if (threadIdx.x < kTile && c0 + threadIdx.x < a.cols) {
        const int64_t tile_y = r0 / kTile;
        const uint32_t byte = scale_byte(SQUARE ? most : col_max[threadIdx.x]);
        reinterpret_cast<uint8_t *>(a.scales_t + (tile_y >> 2) * a.cols + c0 + threadIdx.x)[tile_y & 3] =
            static_cast<uint8_t>(byte);
    }
}

}  // namespace

hipError_t launch_quantize(const QuantArgs &a, int dtype, bool square, hipStream_t s) {
    const uint64_t tiles_x = (a.cols + kTile - 1) / kTile;
    const uint64_t blocks = tiles_x * ((a.rows + kTile - 1) / kTile);
    if (blocks > 0xffffffffull / kBlock) return hipErrorInvalidConfiguration;
    const uint32_t n = static_cast<uint32_t>(blocks), tx = static_cast<uint32_t>(tiles_x);
    if (dtype == PS_F32) {
        if (square) quantize_tile<PS_F32, true><<<n, kBlock, 0, s>>>(a, tx);
        else quantize_tile<PS_F32, false><<<n, kBlock, 0, s>>>(a, tx);
    } else {
        if (square) quantize_tile<PS_BF16, true><<<n, kBlock, 0, s>>>(a, tx);
        else quantize_tile<PS_BF16, false><<<n, kBlock, 0, s>>>(a, tx);
    }
    return hipGetLastError();
}

}  // namespace gadei::learner
