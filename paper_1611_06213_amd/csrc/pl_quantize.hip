// Matrices to 8-bit floating point with a power-of-two scale per block of 128.
//
// Mathematics: e = the least whole number >= -126 with max|x| <= 448 * 2^e over a block's
// finite elements; element = x * 2^-e rounded to nearest even e4m3. 448 = 1.75 * 2^8, so
// e comes from the bits of the maximum: its exponent field once the mantissa is
// rounded up past 1.75, less 8. x * 2^-e is exact unless it falls below fp32's
// smallest numbers, far below e4m3's.
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
constexpr int kRows = 8;   // a thread's rows: threadIdx / 16 + 16 i
constexpr int kPitch = kTile + 4;   // of the transposed tile: whole words, rows in other banks

// The scale's byte (exponent + 127) for the largest finite |x| of a block, as its bits.
__device__ __forceinline__ uint32_t scale_byte(uint32_t bits) {
    const uint32_t e = (bits + 0x1fffffu) >> 23;
    return e < 9 ? 1 : e - 8;
}

// Bits of |x|, 0 for NaN and infinities. Bits of finite numbers compare as they do.
__device__ __forceinline__ uint32_t finite_bits(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0;
}

__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return static_cast<uint32_t>(w);
}

// x * 2^(127 - byte); infinities become NaN (e4m3 has none)
__device__ __forceinline__ float scaled(float x, uint32_t byte) {
    const float up = __uint_as_float((254u - byte) << 23);   // byte is 1 .. 247
    return (__float_as_uint(x) & 0x7fffffffu) == 0x7f800000u ? __uint_as_float(0x7fc00000u) : x * up;
}

template <int X, bool SQUARE>
__global__ __launch_bounds__(kBlock) void quantize_tile(QuantArgs a, uint32_t tiles_x) {
    __shared__ uint32_t col_max[kTile];
    __shared__ uint32_t bytes[kTile * kPitch / 4];   // transposed tile, four rows a word
    __shared__ uint32_t all_max;
    const int64_t r0 = static_cast<int64_t>(blockIdx.x / tiles_x) * kTile;
    const int64_t tile_x = blockIdx.x % tiles_x, c0 = tile_x * kTile;
    const int g = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t col = c0 + 8 * g;
    const int count = a.cols - col >= 8 ? 8 : a.cols > col ? static_cast<int>(a.cols - col) : 0;
    const bool transposed = a.values_t != nullptr;

    float x[kRows][8];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        // a thread's rows come in fours, so that four bytes of a column make a word
        const int64_t r = r0 + 4 * y + (i & 3) + 64 * (i >> 2);
        const bool in = r < a.rows;
        if (in && count == 8) widen8<X>(x[i], load8<X>(a.x, r * a.ld + col));
        else load_some<X>(x[i], a.x, r * a.ld + col, in ? count : 0);
    }
    uint32_t row_max[kRows];
    uint32_t most = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        uint32_t m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, finite_bits(x[i][e]));
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(m, d)));
        row_max[i] = m;
        most = max(most, m);
    }
    if constexpr (SQUARE) {
        if (threadIdx.x == 0) all_max = 0;
        __syncthreads();
        if (g == 0) atomicMax(&all_max, most);
        __syncthreads();
        most = all_max;
#pragma unroll
        for (int i = 0; i < kRows; ++i) row_max[i] = most;
    }
    const int64_t words = static_cast<int64_t>(tile_x >> 2) * a.rows;   // of scales before this row's
    if (a.values != nullptr) {
        const int64_t ld = (a.cols + 127) / 128 * 128;
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int64_t r = r0 + 4 * y + (i & 3) + 64 * (i >> 2);
            if (r >= a.rows) continue;
            const uint32_t byte = scale_byte(row_max[i]);
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = scaled(x[i][e], byte);
            *reinterpret_cast<u32x2 *>(a.values + r * ld + col) =
                u32x2{four_e4m3(v[0], v[1], v[2], v[3]), four_e4m3(v[4], v[5], v[6], v[7])};
            if (g == 0)
                reinterpret_cast<uint8_t *>(a.scales + words + r)[tile_x & 3] = static_cast<uint8_t>(byte);
        }
    }
    if (!transposed) return;

    uint32_t col_bits[8];
    if constexpr (SQUARE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) col_bits[e] = most;
    } else {
        if (threadIdx.x < kTile) col_max[threadIdx.x] = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < kRows; ++i) m = max(m, finite_bits(x[i][e]));
            // the wave's four rows of lanes
            m = max(m, static_cast<uint32_t>(__shfl_xor(m, 16)));
            m = max(m, static_cast<uint32_t>(__shfl_xor(m, 32)));
            if ((threadIdx.x & 63) < 16) atomicMax(&col_max[8 * g + e], m);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) col_bits[e] = col_max[8 * g + e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t byte = scale_byte(col_bits[e]);
#pragma unroll
        for (int h = 0; h < kRows / 4; ++h)
            bytes[((8 * g + e) * kPitch + 4 * y + 64 * h) / 4] =
                four_e4m3(scaled(x[4 * h][e], byte), scaled(x[4 * h + 1][e], byte),
                          scaled(x[4 * h + 2][e], byte), scaled(x[4 * h + 3][e], byte));
    }
    __syncthreads();
    const int64_t ld_t = (a.rows + 127) / 128 * 128;
    // 128 columns of x, 128 bytes each: 32 words a column
    for (int i = threadIdx.x; i < kTile * 32; i += kBlock) {
        const int c = i >> 5, w = i & 31;
        if (c0 + c < a.cols)
            *reinterpret_cast<uint32_t *>(a.values_t + (c0 + c) * ld_t + r0 + 4 * w) =
                bytes[c * (kPitch / 4) + w];
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
