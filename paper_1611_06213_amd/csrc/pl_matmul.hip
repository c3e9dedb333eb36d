// Products of matrices in 8-bit floating point: out = a b^T, a (m x k) and b (n x k) with a
// power-of-two scale per row and block of 128 columns.
//
// Mathematics: out[i, j] = sum over blocks of 2^(ea + eb) * sum over the block's 128
// products, added up in fp32, by one of two instructions:
//
// out in bf16  16 x 16 x 128 on 8-bit operands, which takes the scales of its operands' rows
//              with them (four bytes a row, one per 32 columns; here all four are the block's),
//              so scaling costs no vector work and no second accumulator. It adds products
//              in groups of eight, of which it keeps 13 bits below the largest (measured, as
//              for the 16 x 16 x 32 form): an error of 2^-19 of the sum of the products'
//              magnitudes, root mean square, far below bf16's 2^-9 of the result.
// out in fp32  16 x 16 x 32 on bf16 operands, at half the rate. An 8-bit value times its block's
//              scale is a bf16 number exactly (one conversion instruction for two of them), and
//              this instruction's sums are fp32 sums (an error of 2^-27 or less, measured).
//
// The first operand is b: then a lane holds four neighbouring columns of out, of one row.
// Lane l gives row l % 16 of either operand, and 32 of the block's columns; which 32 does not
// matter as long as both operands agree, since a block's columns share their scale.
//
// Two kernels: `tiles` stages tiles of both operands in LDS, for many rows of a; `slim`, for
// at most 64 rows of a, reads b, by far the larger operand, straight into registers.
// Where there are too few tiles to fill the card, k is split over workgroups; the parts'
// sums go to the workspace and `join` adds them up in order.
#include "pl_device.h"

namespace gadei::learner {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 32 columns of a row of an operand, as the instruction takes them; `scale` holds the block's
// byte in its lowest.
template <bool WIDE> struct Operand;
template <> struct Operand<false> {
    i32x8 v;
    uint32_t scale;
    __device__ __forceinline__ void set(i32x4 x, i32x4 y, uint32_t s) {
        v = i32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        scale = s;
    }
};
template <> struct Operand<true> {
    bf16x8 v[4];
    __device__ __forceinline__ void set(i32x4 x, i32x4 y, uint32_t s) {
        const float two = __uint_as_float((s & 0xffu) << 23);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int lo = i < 2 ? x[2 * i] : y[2 * i - 4], hi = i < 2 ? x[2 * i + 1] : y[2 * i - 3];
            const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, two, false);
            const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, two, true);
            const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, two, false);
            const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, two, true);
            v[i] = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        }
    }
};

__device__ __forceinline__ f32x4 mfma(const Operand<false> &b, const Operand<false> &a, f32x4 c) {
    // formats 0, 0: both e4m3
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b.v, a.v, c, 0, 0, 0, b.scale, 0, a.scale);
}

__device__ __forceinline__ f32x4 mfma(const Operand<true> &b, const Operand<true> &a, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
}

// What becomes of a sum: four columns from n on of row m.
template <int OUT>
__device__ __forceinline__ void finish(const MatmulArgs &g, f32x4 v, uint32_t m, uint32_t n) {
    const int64_t at = m * g.out_ld + n;
    float x[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = v[e];
        if (g.bias != nullptr && n + e < g.n)
            x[e] += g.bias_bf16 ? load1<PS_BF16>(g.bias, n + e) : load1<PS_F32>(g.bias, n + e);
        if (g.relu) x[e] = x[e] < 0.0f ? 0.0f : x[e];   // NaN stays
        if (g.accumulate && n + e < g.n) x[e] += load1<OUT>(g.out, at + e);
    }
    if (n + 4 <= g.n) {
        if constexpr (OUT == PS_F32)
            *reinterpret_cast<f32x4_any *>(static_cast<float *>(g.out) + at) =
                f32x4{x[0], x[1], x[2], x[3]};
        else
            *reinterpret_cast<u32x2_any *>(static_cast<uint16_t *>(g.out) + at) =
                u32x2{bf16x2_rne(x[0], x[1]), bf16x2_rne(x[2], x[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < g.n) store1<OUT>(g.out, at + e, x[e]);
    }
}

// The same for a part of k: to the workspace, whose rows are padded to fours.
__device__ __forceinline__ void keep(const MatmulArgs &g, f32x4 v, uint32_t part, uint32_t m,
                                     uint32_t n) {
    const uint64_t ld = (g.n + 3ull) & ~3ull;
    *reinterpret_cast<f32x4 *>(g.partial + (static_cast<uint64_t>(part) * g.m + m) * ld + n) = v;
}

typedef __attribute__((address_space(1))) uint32_t GlobalWord;
typedef __attribute__((address_space(3))) uint32_t LdsWord;

struct Split {
    uint32_t tiles_m, tiles_n;
    uint32_t parts, steps;   // of k: number of parts, blocks of 128 of each
};

// ------------------------------------------------------------------- tiles

// BM x BN tiles of out by WM x WN waves.
template <int BM, int BN, int WM, int WN, int OUT>
__global__ __launch_bounds__(64 * WM * WN) void tiles(MatmulArgs g, Split sp) {
    constexpr int kWaves = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    constexpr int kLoads = (BM + BN) / 8 / kWaves;   // a wave loads 8 rows of 128 bytes at once
    static_assert((BM + BN) % (8 * kWaves) == 0 && BM % (8 * kLoads) == 0, "whole loads");
    // two buffers that the compiler can tell apart
    __shared__ __attribute__((aligned(128))) uint8_t even[(BM + BN) * 128];
    __shared__ __attribute__((aligned(128))) uint8_t odd[(BM + BN) * 128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t tile = blockIdx.x % (sp.tiles_m * sp.tiles_n);
    const uint32_t part = blockIdx.x / (sp.tiles_m * sp.tiles_n);
    const uint32_t m0 = tile % sp.tiles_m * BM, n0 = tile / sp.tiles_m * BN;
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const uint32_t first = part * sp.steps;
    const uint32_t last = min(blocks, first + sp.steps);   // first < last, as the host splits

    // Rows of the tile: BM of a, then BN of b; rows past the matrix repeat its last. Byte c of
    // row r lies at 128 r + 16 ((c / 16) ^ (r % 8)) + c % 16, so that the rows that lanes read
    // together lie in different banks.
    const bool of_a = wave * kLoads * 8 < BM;
    const uint8_t *base = of_a ? g.a + static_cast<uint64_t>(m0) * ld : g.b + static_cast<uint64_t>(n0) * ld;
    uint32_t from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const uint32_t r = (wave * kLoads + i) * 8 + (lane >> 3);
        const uint32_t row = of_a ? min(r, g.m - 1 - m0) : min(r - BM, g.n - 1 - n0);
        from[i] = row * ld + (((lane & 7) ^ (lane >> 3)) << 4);
    }
    auto fetch = [&](uint8_t *to, uint32_t block) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_global_load_lds(
                (const GlobalWord *)(base + static_cast<uint64_t>(block) * 128 + from[i]),
                (LdsWord *)(to + (wave * kLoads + i) * 1024), 16, 0, 0);
    };

    const int wm = wave % WM * (BM / WM), wn = wave / WM * (BN / WN);
    const int q = lane >> 4, r16 = lane & 15;
    const int low = r16 * 128 + (((2 * q) ^ (r16 & 7)) << 4);
    const int high = r16 * 128 + (((2 * q + 1) ^ (r16 & 7)) << 4);
    uint32_t sa[FM], sb[FN];
    auto scales = [&](uint32_t block) {   // four blocks' at once
        const uint32_t *pa = g.sa + static_cast<uint64_t>(block >> 2) * g.m;
        const uint32_t *pb = g.sb + static_cast<uint64_t>(block >> 2) * g.n;
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = pa[min(m0 + wm + 16 * i + r16, g.m - 1)];
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] = pb[min(n0 + wn + 16 * j + r16, g.n - 1)];
        const int skip = 8 * (block & 3);
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] >>= skip;
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] >>= skip;
    };
    f32x4 acc[FM][FN] = {};
    auto multiply = [&](const uint8_t *at) {
        Operand<OUT == PS_F32> fa, fb[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint8_t *p = at + (BM + wn + 16 * j) * 128;
            fb[j].set(*reinterpret_cast<const i32x4 *>(p + low),
                      *reinterpret_cast<const i32x4 *>(p + high), sb[j]);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const uint8_t *p = at + (wm + 16 * i) * 128;
            fa.set(*reinterpret_cast<const i32x4 *>(p + low),
                   *reinterpret_cast<const i32x4 *>(p + high), sa[i]);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma(fb[j], fa, acc[i][j]);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] >>= 8;
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] >>= 8;
    };
    auto arrived = [] {   // this wave's loads to LDS, then everyone's
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    fetch(even, first);
    scales(first);
    arrived();
    for (uint32_t block = first; block < last; block += 2) {
        if (block + 1 < last) fetch(odd, block + 1);
        if (block != first && (block & 3) == 0) scales(block);
        multiply(even);
        arrived();
        if (block + 1 >= last) break;
        if (block + 2 < last) fetch(even, block + 2);
        if (((block + 1) & 3) == 0) scales(block + 1);
        multiply(odd);
        arrived();
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const uint32_t m = m0 + wm + 16 * i + r16;
        if (m >= g.m) continue;
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const uint32_t n = n0 + wn + 16 * j + 4 * q;
            if (n >= g.n) continue;
            if (sp.parts == 1) finish<OUT>(g, acc[i][j], m, n);
            else keep(g, acc[i][j], part, m, n);
        }
    }
}

// -------------------------------------------------------------------- slim

// 16 rows of b (columns of out) and up to 16 FM rows of a; the four waves of a workgroup take
// the blocks of its part of k in turn and add up their sums in LDS.
constexpr int kSlimWaves = 4;

template <int FM, int OUT>
__global__ __launch_bounds__(64 * kSlimWaves) void slim(MatmulArgs g, Split sp) {
    __shared__ f32x4 sums[kSlimWaves][FM][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int q = lane >> 4, r16 = lane & 15;
    const uint32_t n0 = blockIdx.x % sp.tiles_n * 16, part = blockIdx.x / sp.tiles_n;
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const uint32_t first = part * sp.steps, last = min(blocks, first + sp.steps);
    const uint32_t rb = min(n0 + r16, g.n - 1);
    const uint8_t *pb = g.b + static_cast<uint64_t>(rb) * ld + 32 * q;
    const uint8_t *pa[FM];
    uint32_t ra[FM];
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        ra[i] = min(16u * i + r16, g.m - 1);
        pa[i] = g.a + static_cast<uint64_t>(ra[i]) * ld + 32 * q;
    }
    f32x4 acc[FM] = {};
    constexpr int kAhead = 4;   // blocks whose loads are issued together
    for (uint32_t block = first + wave; block < last; block += kSlimWaves * kAhead) {
        i32x4 b[kAhead][2], a[kAhead][FM][2];
        uint32_t sb[kAhead], sa[kAhead][FM];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint32_t at = min(block + j * kSlimWaves, last - 1);
            const i32x4 *p = reinterpret_cast<const i32x4 *>(pb + static_cast<uint64_t>(at) * 128);
            b[j][0] = __builtin_nontemporal_load(p);
            b[j][1] = __builtin_nontemporal_load(p + 1);
            sb[j] = g.sb[static_cast<uint64_t>(at >> 2) * g.n + rb] >> (8 * (at & 3));
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const i32x4 *pi = reinterpret_cast<const i32x4 *>(pa[i] + static_cast<uint64_t>(at) * 128);
                a[j][i][0] = pi[0];
                a[j][i][1] = pi[1];
                sa[j][i] = g.sa[static_cast<uint64_t>(at >> 2) * g.m + ra[i]] >> (8 * (at & 3));
            }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (block + j * kSlimWaves >= last) break;
            Operand<OUT == PS_F32> fb, fa;
            fb.set(b[j][0], b[j][1], sb[j]);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                fa.set(a[j][i][0], a[j][i][1], sa[j][i]);
                acc[i] = mfma(fb, fa, acc[i]);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (int i = wave; i < FM; i += kSlimWaves) {
        f32x4 v = sums[0][i][lane];
#pragma unroll
        for (int w = 1; w < kSlimWaves; ++w) v += sums[w][i][lane];
        const uint32_t m = 16 * i + r16, n = n0 + 4 * q;
        if (m >= g.m || n >= g.n) continue;
        if (sp.parts == 1) finish<OUT>(g, v, m, n);
        else keep(g, v, part, m, n);
    }
}

// -------------------------------------------------------------------- join

template <int OUT>
__global__ __launch_bounds__(256) void join(MatmulArgs g, uint32_t parts) {
    const uint32_t fours = (g.n + 3) / 4;
    const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<uint64_t>(g.m) * fours) return;
    const uint32_t m = static_cast<uint32_t>(i / fours), n = static_cast<uint32_t>(i % fours) * 4;
    const f32x4 *p = reinterpret_cast<const f32x4 *>(g.partial) + i;
    const uint64_t stride = static_cast<uint64_t>(g.m) * fours;
    f32x4 v = {0, 0, 0, 0};
    for (uint32_t s = 0; s < parts; ++s) v += p[s * stride];
    finish<OUT>(g, v, m, n);
}

// k = 0: sums of no terms.
template <int OUT>
__global__ __launch_bounds__(256) void empty(MatmulArgs g) {
    const uint32_t fours = (g.n + 3) / 4;
    const uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i >= static_cast<uint64_t>(g.m) * fours) return;
    finish<OUT>(g, f32x4{0, 0, 0, 0}, static_cast<uint32_t>(i / fours),
                static_cast<uint32_t>(i % fours) * 4);
}

// ---------------------------------------------------------------- choices

constexpr uint32_t kSlimRows = 64;
constexpr uint32_t kMinSteps = 4;   // blocks of k that a part has at least

struct Choice {
    int bm, bn;
    Split split;
};

Choice choose(uint64_t m, uint64_t n, uint64_t k, bool wide) {
    Choice c{};
    const uint64_t blocks = (k + 127) / 128;
    if (m <= kSlimRows) {
        c.bm = static_cast<int>(m);
        c.bn = 16;
    } else {
        c.bm = c.bn = 128;
    }
    c.split.tiles_m = m <= kSlimRows ? 1 : static_cast<uint32_t>((m + c.bm - 1) / c.bm);
    c.split.tiles_n = static_cast<uint32_t>((n + c.bn - 1) / c.bn);
    // parts of k until every compute unit has a workgroup
    const uint64_t tiles = static_cast<uint64_t>(c.split.tiles_m) * c.split.tiles_n;
    const uint64_t wanted = m <= kSlimRows ? 2 * kCus : kCus;
    uint64_t parts = tiles == 0 ? 1 : wanted / tiles;
    parts = parts < 1 ? 1 : parts;
    const uint64_t least = m <= kSlimRows ? kMinSteps * kSlimWaves : kMinSteps;
    if (parts > blocks / least) parts = blocks / least < 1 ? 1 : blocks / least;
    c.split.steps = static_cast<uint32_t>((blocks + parts - 1) / parts);
    if (c.split.steps == 0) c.split.steps = 1;
    c.split.parts = static_cast<uint32_t>((blocks + c.split.steps - 1) / c.split.steps);
    if (c.split.parts < 1) c.split.parts = 1;
    return c;
}

template <int OUT>
hipError_t launch(const MatmulArgs &g, hipStream_t s) {
    const uint64_t fours = static_cast<uint64_t>(g.m) * ((g.n + 3) / 4);
    const uint64_t join_blocks = (fours + 255) / 256;
    const Choice c = choose(g.m, g.n, g.k, OUT == PS_F32);
    const uint64_t grid = static_cast<uint64_t>(c.split.tiles_m) * c.split.tiles_n * c.split.parts;
    if (join_blocks > 0xffffffffull / 256 || grid > 0xffffffffull / 512)
        return hipErrorInvalidConfiguration;
    const uint32_t blocks = static_cast<uint32_t>(grid);
    if (g.k == 0) {
        empty<OUT><<<static_cast<uint32_t>(join_blocks), 256, 0, s>>>(g);
        return hipGetLastError();
    }
    if (g.m <= 16) slim<1, OUT><<<blocks, 64 * kSlimWaves, 0, s>>>(g, c.split);
    else if (g.m <= 32) slim<2, OUT><<<blocks, 64 * kSlimWaves, 0, s>>>(g, c.split);
    else if (g.m <= kSlimRows) slim<4, OUT><<<blocks, 64 * kSlimWaves, 0, s>>>(g, c.split);
    else tiles<128, 128, 2, 2, OUT><<<blocks, 256, 0, s>>>(g, c.split);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || c.split.parts == 1) return e;
    join<OUT><<<static_cast<uint32_t>(join_blocks), 256, 0, s>>>(g, c.split.parts);
    return hipGetLastError();
}

}  // namespace

size_t matmul_workspace(int64_t m, int64_t n, int64_t k, int out_dtype) {
    if (m == 0 || n == 0 || k == 0) return 0;
    const Choice c = choose(m, n, k, out_dtype == PS_F32);
    if (c.split.parts == 1) return 0;
    return sizeof(float) * size_t(c.split.parts) * size_t(m) * ((size_t(n) + 3) & ~size_t(3));
}

hipError_t launch_matmul(const MatmulArgs &a, int out_dtype, hipStream_t s) {
    return out_dtype == PS_F32 ? launch<PS_F32>(a, s) : launch<PS_BF16>(a, s);
}

}  // namespace gadei::learner
