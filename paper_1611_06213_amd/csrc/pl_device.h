// What the kernels of a learner's operators share: element loads and stores of fp32 and
// bf16 from any element boundary, and the numbers of dropout.
#pragma once

#include <hip/hip_runtime.h>

#include "pl_kernels.h"

namespace gadei::learner {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
// gfx950 loads and stores 16 bytes from any address in one instruction
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

template <int DT>
constexpr int kBytes = DT == PS_F32 ? 4 : 2;

// One dimension of a launch takes fewer than 2^32 threads: more workgroups go on in the second, in rows
// of kGridRow, the last of which may run past the work.
constexpr uint32_t kGridRow = 1u << 20;

inline bool grid_of(uint64_t blocks, uint32_t threads, dim3 *grid) {
    if (blocks > 0xffffffffull - kGridRow) return false;
    if (blocks <= 0xffffffffull / threads) *grid = dim3(static_cast<uint32_t>(blocks));
    else *grid = dim3(kGridRow, static_cast<uint32_t>((blocks + kGridRow - 1) / kGridRow));
    return true;
}

__device__ __forceinline__ uint32_t block_index() { return blockIdx.x + blockIdx.y * kGridRow; }

// Bytes of a result that are left in the caches (256 MB of last level) for whoever reads it.
constexpr uint64_t kCached = 64ull << 20;

// bf16 -> fp32 is exact: the bf16 bits are the upper half of the fp32 bits
__device__ __forceinline__ float lo_bf16(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float hi_bf16(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// two fp32 values rounded to nearest even bf16, a in the low half
__device__ __forceinline__ uint32_t bf16x2_rne(float a, float b) {
    const f32x2 x = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// Eight consecutive elements as loaded: 16 bytes of bf16, or 32 of fp32.
template <int DT> struct Bits8;
template <> struct Bits8<PS_F32> { f32x4 a, b; };
template <> struct Bits8<PS_BF16> { u32x4 a; };

// All eight lie inside the row.
template <int DT>
__device__ __forceinline__ Bits8<DT> load8(const void *p, int64_t i) {
    Bits8<DT> r;
    if constexpr (DT == PS_F32) {
        const f32x4_any *q = reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + i);
        r.a = q[0];
        r.b = q[1];
    } else {
        r.a = *reinterpret_cast<const u32x4_any *>(static_cast<const uint16_t *>(p) + i);
    }
    return r;
}

template <int DT>
__device__ __forceinline__ float load1(const void *p, int64_t i) {
    if constexpr (DT == PS_F32) return static_cast<const float *>(p)[i];
    else return lo_bf16(static_cast<const uint16_t *>(p)[i]);
}

// The first `count` (1..8) of them; the others are 0.
template <int DT>
__device__ __forceinline__ Bits8<DT> load8_some(const void *p, int64_t i, int count) {
    Bits8<DT> r = {};
    if constexpr (DT == PS_F32) {
        const float *q = static_cast<const float *>(p) + i;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (e < count) r.a[e] = q[e];
            if (4 + e < count) r.b[e] = q[4 + e];
        }
    } else {
        const uint16_t *q = static_cast<const uint16_t *>(p) + i;
        uint32_t x[8] = {};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < count) x[e] = q[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) r.a[e] = x[2 * e] | x[2 * e + 1] << 16;
    }
    return r;
}

template <int DT>
__device__ __forceinline__ void widen8(float (&x)[8], const Bits8<DT> &r) {
    if constexpr (DT == PS_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = r.a[e]; x[4 + e] = r.b[e]; }
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[2 * e] = lo_bf16(r.a[e]); x[2 * e + 1] = hi_bf16(r.a[e]); }
    }
}

// The first `count` (1..8) of eight consecutive elements; the others are 0.
template <int DT>
__device__ __forceinline__ void load_some(float (&x)[8], const void *p, int64_t i, int count) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < count ? load1<DT>(p, i + e) : 0.0f;
}

template <int DT>
__device__ __forceinline__ void store1(void *p, int64_t i, float x) {
    if constexpr (DT == PS_F32) static_cast<float *>(p)[i] = x;
    else static_cast<uint16_t *>(p)[i] = static_cast<uint16_t>(bf16x2_rne(x, 0.0f));
}

// NT: not to be kept in the caches.
template <int DT, bool NT = false>
__device__ __forceinline__ void store8(void *p, int64_t i, const float (&x)[8]) {
    if constexpr (DT == PS_F32) {
        f32x4_any *q = reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + i);
        const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        if constexpr (NT) {
            __builtin_nontemporal_store(a, q);
            __builtin_nontemporal_store(b, q + 1);
        } else {
            q[0] = a;
            q[1] = b;
        }
    } else {
        u32x4_any *q = reinterpret_cast<u32x4_any *>(static_cast<uint16_t *>(p) + i);
        const u32x4 a = {bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3]), bf16x2_rne(x[4], x[5]),
                         bf16x2_rne(x[6], x[7])};
        if constexpr (NT) __builtin_nontemporal_store(a, q);
        else *q = a;
    }
}

// store8 past the caches by all 64 lanes of a wave, whose elements are 512 neighbours: lane l's
// begin at i = first + 8 l. Stores past the caches should fill whole lines, and those of fp32, 16 of
// a lane's 32 bytes at a time, would not: they go through `stage`, 2 KB of LDS of the wave's own.
// (The gradient of an embedding from 32768 tokens of 4096 bf16 columns into 536 MB of fp32 rows:
// 208 us with plain stores, 165 so.)
template <int DT>
__device__ __forceinline__ void store8_lines(void *p, int64_t i, const float (&x)[8], f32x4 *stage) {
    if constexpr (DT == PS_F32) {
        const int lane = threadIdx.x & 63;
        stage[2 * lane] = f32x4{x[0], x[1], x[2], x[3]};
        stage[2 * lane + 1] = f32x4{x[4], x[5], x[6], x[7]};
        __builtin_amdgcn_wave_barrier();
        const f32x4 a = stage[lane], b = stage[64 + lane];
        __builtin_amdgcn_wave_barrier();
        float *q = static_cast<float *>(p) + i - 4 * lane;
        __builtin_nontemporal_store(a, reinterpret_cast<f32x4_any *>(q));
        __builtin_nontemporal_store(b, reinterpret_cast<f32x4_any *>(q + 256));
    } else {
        store8<DT, true>(p, i, x);
    }
}

template <int DT>
__device__ __forceinline__ void store_some(void *p, int64_t i, const float (&x)[8], int count) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < count) store1<DT>(p, i + e, x[e]);
}

// Philox4x32-10: the four words for columns 8 * group .. + 7 of `row`. Ten rounds of
// two 32 x 32 -> 64-bit products; the keys are the same for the whole launch and
// stay in scalar registers.
__device__ __forceinline__ u32x4 philox(uint32_t group, uint32_t row, const Drop &d) {
    uint32_t c0 = group, c1 = row, c2 = d.o0, c3 = d.o1, k0 = d.k0, k1 = d.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = static_cast<uint64_t>(0xD2511F53u) * c0;
        const uint64_t p1 = static_cast<uint64_t>(0xCD9E8D57u) * c2;
        c0 = static_cast<uint32_t>(p1 >> 32) ^ c1 ^ k0;
        c2 = static_cast<uint32_t>(p0 >> 32) ^ c3 ^ k1;
        c1 = static_cast<uint32_t>(p1);
        c3 = static_cast<uint32_t>(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// Eight elements of columns 8 * group .. + 7 times `factor`, the dropped ones 0.
__device__ __forceinline__ void drop8(float (&x)[8], float factor, uint32_t group, uint32_t row,
                                      const Drop &d) {
    const u32x4 w = philox(group, row, d);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t number = e & 1 ? w[e >> 1] >> 16 : w[e >> 1] & 0xffffu;
        x[e] = number >= d.drop ? x[e] * factor : 0.0f;
    }
}

}  // namespace gadei::learner
