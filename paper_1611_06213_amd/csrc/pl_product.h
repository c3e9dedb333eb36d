// What the products of a learner's operators share (pl_matmul.hip, pl_matmul_int8.hip): rows of
// operands by buffer loads, tiles and parts of k as work units, results in whole lines.
#pragma once

#include "pl_device.h"

namespace gadei::learner {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four columns from n on of the row that begins at element `row`; zeros from column `end` on.
template <int DT>
__device__ __forceinline__ f32x4 load4(const void *p, int64_t row, uint32_t n, uint32_t end) {
    f32x4 v = {0, 0, 0, 0};
    if (n + 4 <= end) {
        if constexpr (DT == PS_F32) {
            v = *reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + row + n);
        } else {
            const u32x2 w = *reinterpret_cast<const u32x2_any *>(static_cast<const uint16_t *>(p) + row + n);
            v = f32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u),
                      __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < end) v[e] = load1<DT>(p, row + n + e);
    }
    return v;
}

// 16 bytes of row m's results from column n on; edge: some may lie past the last column.
template <class T, class Args>
__device__ __forceinline__ void put(const Args &g, u32x4 w, uint32_t m, uint32_t n, bool edge) {
    constexpr uint32_t N = 16 / sizeof(T);
    T *to = static_cast<T *>(g.out) + m * g.out_ld + n;
    if (!edge || n + N <= g.n) {
        *reinterpret_cast<u32x4_any *>(to) = w;
    } else {
#pragma unroll
        for (uint32_t c = 0; c < N; ++c) {
            if (n + c >= g.n) continue;
            if constexpr (sizeof(T) == 4) to[c] = __uint_as_float(w[c]);
            else to[c] = static_cast<T>(w[c / 2] >> (16 * (c % 2)));
        }
    }
}

// Lanes 16 .. 31 and 48 .. 63 of a for lanes 0 .. 15 and 32 .. 47 of b.
__device__ __forceinline__ void swap_rows(u32x4 &a, u32x4 &b) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const auto p = __builtin_amdgcn_permlane16_swap(a[c], b[c], false, false);
        a[c] = p[0];
        b[c] = p[1];
    }
}

// A run of memory that is read by 32-bit offsets: a lane's own, and one that all lanes share
// (which costs no vector register). What lies outside reads as zero.
struct Buffer {
    __amdgpu_buffer_rsrc_t rsrc;
    Buffer() = default;
    __device__ __forceinline__ Buffer(const void *p, uint32_t bytes)
        : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, static_cast<int>(bytes),
                                                 0x27000)) {}
    static constexpr uint32_t kOutside = 0x80000000u;   // of every buffer
    // 16 bytes a lane, to LDS at 16 bytes a lane
    __device__ __forceinline__ void to_lds(uint8_t *to, uint32_t lane, uint32_t shared) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(
            rsrc, (__attribute__((address_space(3))) void *)to, 16, lane, shared, 0, 0);
    }
    // four bytes a lane
    __device__ __forceinline__ void words_to_lds(void *to, uint32_t lane) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void *)to, 4, lane, 0,
                                                 0, 0);
    }
    __device__ __forceinline__ i32x4 sixteen(uint32_t lane, uint32_t shared) const {
        return __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane, shared, 0));
    }
    __device__ __forceinline__ uint32_t word(uint32_t lane) const {
        return __builtin_amdgcn_raw_buffer_load_b32(rsrc, lane, 0, 0);
    }
    __device__ __forceinline__ uint32_t half(uint32_t lane) const {
        return static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(rsrc, lane, 0, 0));
    }
};

struct Split {
    uint32_t tiles_m, tiles_n;
    uint32_t parts, steps;   // of k: number of parts, blocks of 128 of each
};

// Which tile of which part of k the work unit `unit` is. Workgroups go round the eight XCDs, each
// with an L2 of its own: an XCD takes a contiguous run of an order that walks bands of eight rows
// of tiles column by column, so that the 32 tiles that its compute units work on share their rows
// of a and b.
__device__ __forceinline__ void place(const Split &sp, uint32_t unit, uint32_t *tile_m, uint32_t *tile_n,
                                      uint32_t *part) {
    constexpr uint32_t kXcds = 8, kBand = 8;
    const uint32_t tiles = sp.tiles_m * sp.tiles_n, all = tiles * sp.parts;
    const uint32_t xcd = unit % kXcds, each = all / kXcds, more = all % kXcds;
    const uint32_t t = xcd * each + min(xcd, more) + unit / kXcds;
    *part = t / tiles;
    const uint32_t in = t % tiles, band = in / (kBand * sp.tiles_n), at = in % (kBand * sp.tiles_n);
    const uint32_t height = min(kBand, sp.tiles_m - band * kBand);
    *tile_m = band * kBand + at % height;
    *tile_n = at / height;
}

}  // namespace gadei::learner
