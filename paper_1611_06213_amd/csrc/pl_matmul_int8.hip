// Products of matrices of 8-bit integers with a scale for each row of either: out = (a b^T) scaled,
// a (m x k), a row a token, and b (n x k), a row a channel.
//
// Mathematics: a row's scale is s = max(most, 2^-100) / 127 with most = max|row|, its integers are
// round(x (127 (1 / max(most, 2^-100)))); out[i, j] = (sum over k of qa qb) sa[i] sb[j]. The sums are
// exact: |sum| <= 127^2 k < 2^31 up to k = 2^17. So how k is split, and the order of the parts,
// cannot be seen in a result. A row with a NaN or an infinity has the scale NaN.
//
// The instructions take 16 bytes of 32 (16) rows of either operand a lane, 32 (64) columns in all;
// which of the columns a lane holds does not matter as long as both operands agree. The first
// operand is b: then a lane holds four neighbouring columns of out, of one row.
//
// Two kernels: `tiles` stages tiles of both operands in LDS, for many rows of a; `slim`, for at most
// 64 rows of a, reads b straight into registers. Where there are too few tiles to fill the card, k is
// split over workgroups; the parts' sums go to the workspace and `join` adds them up.
//
// 8192 x 8192 x 8192 to bf16 takes 466 us (2.4 POP/s; bound by matrix pipes and the clock that power
// allows: 430 in the first call, to 600 where calls follow one another; the library's product, into 32-bit sums,
// 451, 445 and to 580 in turn with it), 1 x 4096 x 25088 21 us (103 MB, 4.9 TB/s; bound by reading b), 128 x 4096
// x 9216 15 and 4 for the join (bound by the latency of its first loads and last stores, as a workgroup has 12
// blocks of k).
#include <algorithm>

#include "pl_fp8.h"
#include "pl_product.h"

namespace gadei::learner {
namespace {

// ---------------------------------------------------------------- integers

constexpr float kLeast = 0x1p-100f;   // below it a row's largest would have no inverse in fp32
constexpr int kKept = 4;              // eights of a row that a thread keeps from its maximum to its integers

struct RowScale {
    float scale, inverse;
    __device__ __forceinline__ explicit RowScale(uint32_t most_bits) {
        const float most = max(__uint_as_float(most_bits), kLeast);
        scale = most_bits < 0x7f800000u ? most / 127.0f : __builtin_nanf("");
        inverse = 127.0f * (1.0f / most);
    }
};

// Magnitudes compare as their bits do, those of NaN and infinity above all others.
__device__ __forceinline__ uint32_t most_of(const float (&x)[8], uint32_t m) {
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7fffffffu);
    return m;
}

// Eight integers. The sum with 1.5 * 2^23 rounds to a whole number, nearest even, and has it in its
// low bits.
__device__ __forceinline__ u32x2 integers(const float (&x)[8], float inverse) {
#pragma clang fp contract(off)
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(x[e] * inverse + 12582912.0f);
    u32x2 w;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400);
        const uint32_t hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x04000c0c);
        w[h] = lo | hi;
    }
    return w;
}

template <int X>
__device__ __forceinline__ void row8(float (&x)[8], const void *p, int64_t at, int count) {
    widen8<X>(x, count == 8 ? load8<X>(p, at) : load8_some<X>(p, at, count));
}

__device__ __forceinline__ int count_at(int64_t cols, int64_t col) {
    return cols - col >= 8 ? 8 : cols > col ? static_cast<int>(cols - col) : 0;
}

__device__ __forceinline__ uint32_t most_of_wave(uint32_t m) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(m, d)));
    return m;
}

// A row a wave (threadIdx.y) or a row a workgroup. Bound by memory: 8192 x 8192 bf16 32 to 40 us (201 MB,
// 5.0 to 6.3 TB/s).
template <int X, int THREADS>
__global__ __launch_bounds__(THREADS) void quantize(Int8QuantArgs a) {
    constexpr int kWaves = THREADS / 64;
    __shared__ uint32_t lds[kWaves];
    const int64_t row = static_cast<int64_t>(block_index()) * blockDim.y + threadIdx.y;
    if (row >= a.rows) return;   // a whole wave, or a whole workgroup
    const int64_t ld = (a.cols + 127) / 128 * 128, step = 8 * blockDim.x, first = 8 * threadIdx.x;
    float x[kKept][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kKept; ++i) {
        const int64_t col = first + i * step;
        row8<X>(x[i], a.x, row * a.ld + col, count_at(a.cols, col));
        m = most_of(x[i], m);
    }
    for (int64_t col = first + kKept * step; col < a.cols; col += step) {
        float more[8];
        row8<X>(more, a.x, row * a.ld + col, count_at(a.cols, col));
        m = most_of(more, m);
    }
    m = most_of_wave(m);
    if (blockDim.x > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = max(m, lds[w]);
    }
    const RowScale s(m);
    if (threadIdx.x == 0) a.scales[row] = s.scale;
#pragma unroll
    for (int i = 0; i < kKept; ++i) {
        const int64_t col = first + i * step;
        if (col < ld) *reinterpret_cast<u32x2 *>(a.values + row * ld + col) = integers(x[i], s.inverse);
    }
    for (int64_t col = first + kKept * step; col < ld; col += step) {
        float more[8];
        row8<X>(more, a.x, row * a.ld + col, count_at(a.cols, col));
        *reinterpret_cast<u32x2 *>(a.values + row * ld + col) = integers(more, s.inverse);
    }
}

// ----------------------------------------------------------------- results

// What becomes of four sums: every step rounds by itself, so that all kernels give the same.
__device__ __forceinline__ f32x4 scaled(i32x4 sum, float row_scale, f32x4 scale, f32x4 bias, bool with_bias,
                                        bool relu) {
#pragma clang fp contract(off)
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = static_cast<float>(sum[e]) * row_scale * scale[e];
        if (with_bias) x[e] += bias[e];
        if (relu) x[e] = x[e] < 0.0f ? 0.0f : x[e];   // NaN stays
    }
    return x;
}

// Four columns from n on of row m, from their sums.
template <int OUT>
__device__ __forceinline__ void finish(const Int8Args &g, i32x4 v, float row_scale, uint32_t m, uint32_t n) {
    f32x4 bias = {};
    if (g.bias != nullptr) bias = g.bias_bf16 ? load4<PS_BF16>(g.bias, 0, n, g.n) : load4<PS_F32>(g.bias, 0, n, g.n);
    const f32x4 x = scaled(v, row_scale, load4<PS_F32>(g.sb, 0, n, g.n), bias, g.bias != nullptr, g.relu);
    const int64_t at = m * g.out_ld + n;
    if (n + 4 <= g.n) {
        if constexpr (OUT == PS_F32)
            *reinterpret_cast<f32x4_any *>(static_cast<float *>(g.out) + at) = x;
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
__device__ __forceinline__ void keep(const Int8Args &g, i32x4 v, uint32_t part, uint32_t m, uint32_t n) {
    const uint64_t ld = (g.n + 3ull) & ~3ull;
    *reinterpret_cast<i32x4 *>(g.partial + (static_cast<uint64_t>(part) * g.m + m) * ld + n) = v;
}

// ------------------------------------------------------------------- tiles

// Of s_waitcnt: until so many copies and loads, and reads of LDS, are under way. By the builtin, which tells
// the compiler: it would wait for its reads once more.
constexpr int wait(int vm, int lgkm) { return (vm & 15) | (vm >> 4) << 14 | 7 << 4 | lgkm << 8; }
constexpr int kAnyReads = 15;
constexpr int kSums = -2;   // for OUT: parts' sums

// c += b a^T, with c where it is: from the builtin the compiler makes moves of sums from register to register in
// the loop over k (8192^3 438 us with it, 419 so). It knows nothing of this instruction's time, so `settle`
// comes between it and any other use of c.
__device__ __forceinline__ void mfma(i32x4 &c, const i32x4 &b, const i32x4 &a) {
    asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(c) : "v"(b), "v"(a));
}

// What was written to the sums before this, by products or by moves, is there after it.
template <int F>
__device__ __forceinline__ void settle(i32x4 (&acc)[F][F][2][2]) {
    auto tie = [&] {
#pragma unroll
        for (int i = 0; i < 4 * F * F; ++i) asm volatile("" : "+a"(acc[i / (4 * F)][i / 4 % F][i / 2 % 2][i % 2]));
    };
    tie();
    asm volatile("s_nop 15\n\ts_nop 15");
    tie();
}

// Tiles of 64 F x 64 F by 2 x 2 waves, each F x F times four blocks of 16 x 16.
//
// A step is 64 columns of k. LDS holds four steps of either operand, which copies bring there from
// memory without registers; the registers hold the step that multiplies and the one after it. So in
// step s, step s + 1 is read from LDS, step s + 4 is copied to where s was, and the copies have three
// steps to arrive: at the end of a step all but those of the last two are waited for.
template <int F, int OUT>
__global__ __launch_bounds__(256, F == 2 ? 2 : 1) void tiles(Int8Args g, Split sp) {
    constexpr int B = 64 * F, BYTES = B * 64, N = 2 * F;
    // buffers that the compiler can tell apart: it would wait for all copies before every read of LDS
    // if it could not
    __shared__ __attribute__((aligned(128))) uint8_t a0[BYTES], a1[BYTES], a2[BYTES], a3[BYTES], b0[BYTES],
        b1[BYTES], b2[BYTES], b3[BYTES];
    // of a tile's rows and columns; the next tile's scales are copied while this one's are used
    __shared__ __attribute__((aligned(16))) float row_scales[2 * B], scales[2 * B], biases[B];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const int wm = wave % 2 * (32 * F), wn = wave / 2 * (32 * F);
    const int q = lane >> 4, r16 = lane & 15;

    // A copy takes 16 rows of 64 bytes. Rows past the matrix are outside the buffers' bounds and read
    // as zeros. 16 bytes c of row r lie at 64 r + 16 (c ^ (-r / 4 % 4)), so that the 16 lanes that LDS
    // serves at once (0-3, 12-15, 20-23 and 24-27, and their like) lie in different banks. A lane reads
    // 16 bytes of rows r16 and, 16 rows further, r16 + 16.
    const uint32_t from = (lane >> 2) * ld + (((lane & 3) ^ (-(lane >> 4) & 3)) << 4);
    const int low = r16 * 64 + ((q ^ (-(r16 >> 2) & 3)) << 4), high = low + 16 * 64;

    // a work unit: a tile and a part of k
    uint32_t m0, n0, part, first, last;
    Buffer rows_a, rows_b;
    auto take = [&](uint32_t unit) {
        uint32_t tile_m, tile_n;
        place(sp, unit, &tile_m, &tile_n, &part);
        m0 = tile_m * B;
        n0 = tile_n * B;
        first = part * sp.steps;
        last = min(blocks, first + sp.steps);   // first < last, as the host splits
        rows_a = Buffer(g.a + static_cast<uint64_t>(m0) * ld, min(g.m - m0, uint32_t(B)) * ld);
        rows_b = Buffer(g.b + static_cast<uint64_t>(n0) * ld, min(g.n - n0, uint32_t(B)) * ld);
    };
    // The wave's copies of a step (half 0 or 1 of a block): F of a, F of b. Blocks past the last: no bytes.
    auto copy = [&](uint8_t *a, uint8_t *b, int i, uint32_t block, int half) {
        const uint32_t lanes = block < last ? from : Buffer::kOutside;
        if (i < F)
            rows_a.to_lds(a + (wave * F + i) * 1024, lanes, (wave * F + i) * 16 * ld + block * 128 + half * 64);
        else
            rows_b.to_lds(b + (wave * F + i - F) * 1024, lanes,
                          (wave * F + i - F) * 16 * ld + block * 128 + half * 64);
    };
    // The thread's number outside of the loop over k, computed anew: the compiler would keep what is made
    // of it, and have no registers for that in the loop.
    auto lane_now = [] {
        uint32_t lane;
        asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=&v"(lane));
        return lane;
    };
    uint32_t turn = 0;
    auto begin = [&] {
        if (64 * wave < B) {
            const uint32_t thread = 64 * wave + lane_now(), to = turn * B + 64 * wave;
            Buffer(g.sa, g.m * 4).words_to_lds(row_scales + to, (m0 + thread) * 4);
            Buffer(g.sb, g.n * 4).words_to_lds(scales + to, (n0 + thread) * 4);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < N; ++i) copy(a0, b0, i, first, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) copy(a1, b1, i, first, 1);
#pragma unroll
        for (int i = 0; i < N; ++i) copy(a2, b2, i, first + 1, 0);
#pragma unroll
        for (int i = 0; i < N; ++i) copy(a3, b3, i, first + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
    };

    struct Raw { i32x4 lo, hi; };
    struct Step { Raw a[F], b[F]; };
    i32x4 acc[F][F][2][2];   // of 16 columns and 16 rows of out each
    auto read_a = [&](Step &s, const uint8_t *at, int i) {
        const uint8_t *p = at + (wm + 32 * i) * 64;
        s.a[i] = Raw{*reinterpret_cast<const i32x4 *>(p + low), *reinterpret_cast<const i32x4 *>(p + high)};
    };
    auto read_b = [&](Step &s, const uint8_t *at, int j) {
        const uint8_t *p = at + (wn + 32 * j) * 64;
        s.b[j] = Raw{*reinterpret_cast<const i32x4 *>(p + low), *reinterpret_cast<const i32x4 *>(p + high)};
    };
    // Multiply `now`, read `next` (from a and b), copy half `half` of block `block` to a_to and b_to.
    auto step = [&](const Step &now, Step &next, const uint8_t *a, const uint8_t *b, uint8_t *a_to, uint8_t *b_to,
                    uint32_t block, int half) {
        // Reads and copies one at a time between the products: the memory pipeline takes a copy every
        // 16 cycles from four waves, and a wave that has to wait there issues no products. The reads
        // end early, so that none is waited for at the step's end.
        constexpr int S = F * F;
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const int i = t / F, j = t % F;
#pragma unroll
            for (int hb = 0; hb < 2; ++hb)
#pragma unroll
                for (int ha = 0; ha < 2; ++ha)
                    mfma(acc[i][j][hb][ha], hb ? now.b[j].hi : now.b[j].lo, ha ? now.a[i].hi : now.a[i].lo);
#pragma unroll
            for (int c = t * 3 * N / (2 * S); c < (t + 1) * 3 * N / (2 * S) && c < N; ++c) {
                if (c < F) read_a(next, a, c);
                else read_b(next, b, c - F);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = (t * N + N / 2) / S; c < ((t + 1) * N + N / 2) / S && c < N; ++c)
                copy(a_to, b_to, c, block, half);
            __builtin_amdgcn_sched_barrier(0);
        }
        // This wave's copies but those of the last two steps have arrived, and its reads; then
        // everyone's.
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait(2 * N, 0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    Step x, y;
    auto block = [&](uint32_t k, uint8_t *pa0, uint8_t *pb0, uint8_t *pa1, uint8_t *pb1, uint8_t *pa2,
                     uint8_t *pb2) {
        step(x, y, pa1, pb1, pa0, pb0, k + 2, 0);
        step(y, x, pa2, pb2, pa1, pb1, k + 2, 1);
    };

    uint32_t unit = blockIdx.x;
    asm volatile("; the first unit's copies");
    take(unit);
    begin();
    for (;;) {
        int zero = 0;
        asm volatile("" : "+v"(zero));   // the compiler would keep zeros in registers from unit to unit
#pragma unroll
        for (int i = 0; i < 4 * F * F; ++i)
            acc[i / (4 * F)][i / 4 % F][i / 2 % 2][i % 2] = i32x4{zero, zero, zero, zero};
        settle(acc);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait(2 * N, kAnyReads));   // steps 0 and 1
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < F; ++i) read_a(x, a0, i);
#pragma unroll
        for (int j = 0; j < F; ++j) read_b(x, b0, j);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait(63, 0));
        __builtin_amdgcn_s_barrier();   // a0 and b0 may be written
        asm volatile("" ::: "memory");
        // an odd number of blocks is followed by one of zeros: a loop with a way out in its middle
        // would have the compiler move all sums from register to register
        for (uint32_t k = first; k < last; k += 2) {
            block(k, a0, b0, a1, b1, a2, b2);
            block(k + 1, a2, b2, a3, b3, a0, b0);
        }

        settle(acc);
        // The results go out from the registers, while the next unit's first copies are under way.
        const uint32_t lane1 = lane_now(), thread = 64 * wave + lane1;
        const uint32_t q1 = lane1 >> 4, r1 = lane1 & 15;
        const uint32_t m1 = m0 + wm, n1 = n0 + wn, part1 = part;
        const bool edge = n0 + B > g.n, with_bias = OUT != kSums && g.bias != nullptr;
        unit += gridDim.x;
        const bool more = unit < sp.tiles_m * sp.tiles_n * sp.parts;
        const float *const rows_of = row_scales + turn * B + wm + r1, *const columns_of = scales + turn * B + wn;
        // the bias of the thread's column, zero where there is none: no register holds it through the loop
        const Buffer bias32(g.bias, with_bias && !g.bias_bf16 ? g.n * 4 : 0);
        const Buffer bias16(g.bias, with_bias && g.bias_bf16 ? g.n * 2 : 0);
        const uint32_t bias_word = bias32.word((n0 + thread) * 4);
        const uint32_t bias_half = bias16.half((n0 + thread) * 2);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait(0, 0));   // the last copies write zeros to LDS
        if (thread < B) biases[thread] = __uint_as_float(bias_word | bias_half << 16);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(wait(63, 0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (more) {
            turn ^= 1;
            take(unit);
            begin();
        }
        // a lane holds columns 4 q1 + 0..3 of row r1 of each 16 x 16
#pragma unroll
        for (int j0 = 0; j0 < F; j0 += 2) {   // 64 columns of a row after one another: a line of bf16
#pragma unroll
            for (int ij = 0; ij < 4 * F; ++ij) {
                const int i = ij / 4, ha = ij / 2 % 2, j = j0 + ij % 2;
                const uint32_t to = m1 + 32 * i + 16 * ha + r1, n = n1 + 32 * j;
                f32x4 v[2];
#pragma unroll
                for (int hb = 0; hb < 2; ++hb) {
#pragma clang fp contract(off)
                    // as `scaled` has it, in fewer registers
                    const i32x4 sum = acc[i][j][hb][ha];
                    if constexpr (OUT == kSums) {
                        v[hb] = __builtin_bit_cast(f32x4, sum);
                        continue;
                    }
                    const uint32_t c = 32 * j + 16 * hb + 4 * q1;
                    const f32x4 sb = *reinterpret_cast<const f32x4 *>(columns_of + c);
#pragma unroll
                    for (int d = 0; d < 4; ++d)
                        v[hb][d] = static_cast<float>(sum[d]) * rows_of[32 * i + 16 * ha] * sb[d];
                    if (with_bias) v[hb] += *reinterpret_cast<const f32x4 *>(biases + wn + c);
                    if (g.relu) {
#pragma unroll
                        for (int d = 0; d < 4; ++d) v[hb][d] = v[hb][d] < 0.0f ? 0.0f : v[hb][d];   // NaN stays
                    }
                }
                if (to >= g.m) continue;
                if constexpr (OUT == kSums) {
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb)
                        if (n + 16 * hb + 4 * q1 < g.n)
                            keep(g, __builtin_bit_cast(i32x4, v[hb]), part1, to, n + 16 * hb + 4 * q1);
                } else if constexpr (OUT == PS_F32) {
#pragma unroll
                    for (int hb = 0; hb < 2; ++hb)
                        put<float>(g, __builtin_bit_cast(u32x4, v[hb]), to, n + 16 * hb + 4 * q1, edge);
                } else {
                    // Eights of bf16 first: of the two rows of lanes that hold neighbouring fours, one takes
                    // both of the first sixteen columns, the other both of the second.
                    u32x4 w;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const auto p = __builtin_amdgcn_permlane16_swap(bf16x2_rne(v[0][2 * c], v[0][2 * c + 1]),
                                                                        bf16x2_rne(v[1][2 * c], v[1][2 * c + 1]), false,
                                                                        false);
                        w[c] = p[0];
                        w[2 + c] = p[1];
                    }
                    put<uint16_t>(g, w, to, n + 16 * (q1 & 1) + 4 * (q1 & 2), edge);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!more) break;
    }
}

// -------------------------------------------------------------------- slim

// 16 rows of b (columns of out) a workgroup and up to 16 FM rows of a: bound by reading b, once,
// straight into registers. The waves take the blocks of k in turn, the loads of several blocks under
// way in each, and add up their sums in LDS: no part of k goes through memory.
//
// X >= 0: a is not integers yet but given as x. Every workgroup converts all of it, into LDS, while
// its first rows of b are under way: for few rows that is less than a launch.
constexpr int kGiven = -1;
template <int FM>
constexpr int kAhead = FM == 1 ? 4 : FM == 2 ? 2 : 1;   // blocks whose loads are issued together

template <int FM, int OUT, int X, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void slim(Int8Args g, Split sp) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ uint32_t most[16 * FM];
    constexpr int A = kAhead<FM>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, r16 = lane & 15;
    const uint32_t part = block_index() / sp.tiles_n, n0 = block_index() % sp.tiles_n * 16;
    if (part >= sp.parts) return;
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const uint32_t first = part * sp.steps, last = min(blocks, first + sp.steps);
    const uint32_t pitch = ld + 16;   // of x's rows in LDS: in different banks
    // rows past a matrix, and blocks past the last, read as zeros
    const Buffer rows_b(g.b + static_cast<uint64_t>(n0) * ld, min(g.n - n0, 16u) * ld);
    const Buffer rows_a(g.a, X == kGiven ? g.m * ld : 0);
    const uint32_t from = r16 * ld + 32 * q;

    struct Ahead { i32x4 b[A][2], a[A][FM][2]; } t;
    auto load = [&](uint32_t block) {
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const uint32_t at = block + j * WAVES;
            const uint32_t lanes = at < last ? from : Buffer::kOutside;
            t.b[j][0] = rows_b.sixteen(lanes, at * 128);
            t.b[j][1] = rows_b.sixteen(lanes, at * 128 + 16);
            if constexpr (X == kGiven) {
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    t.a[j][i][0] = rows_a.sixteen(lanes, 16 * i * ld + at * 128);
                    t.a[j][i][1] = rows_a.sixteen(lanes, 16 * i * ld + at * 128 + 16);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // all under way before the first is used
    };
    load(first + wave);
    if constexpr (X != kGiven) {
        if (threadIdx.x < 16 * FM) most[threadIdx.x] = 0;
        __syncthreads();
        // eights of all rows, sixteen lanes a block; the first kKept of a thread stay in registers
        const uint32_t eights = g.m * blocks * 16;
        float kept[kKept][8];
        auto read = [&](float (&x)[8], uint32_t i) {
            const uint32_t m = i / (16 * blocks), col = i % (16 * blocks) * 8;
            row8<X>(x, g.x, m * g.x_ld + col, i < eights ? count_at(g.k, col) : 0);
        };
        auto largest = [&](const float (&x)[8], uint32_t i) {
            uint32_t v = most_of(x, 0);   // sixteen lanes are of one row
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(v, d)));
            if ((threadIdx.x & 15) == 0 && i < eights) atomicMax(&most[i / (16 * blocks)], v);
        };
#pragma unroll
        for (int j = 0; j < kKept; ++j) read(kept[j], threadIdx.x + j * 64 * WAVES);
#pragma unroll
        for (int j = 0; j < kKept; ++j) largest(kept[j], threadIdx.x + j * 64 * WAVES);
        for (uint32_t i = threadIdx.x + kKept * 64 * WAVES; i < eights; i += 64 * WAVES) {
            float x[8];
            read(x, i);
            largest(x, i);
        }
        __syncthreads();
        auto convert = [&](const float (&x)[8], uint32_t i) {
            const uint32_t m = i / (16 * blocks), col = i % (16 * blocks) * 8;
            if (i < eights) *reinterpret_cast<u32x2 *>(lds + m * pitch + col) = integers(x, RowScale(most[m]).inverse);
        };
#pragma unroll
        for (int j = 0; j < kKept; ++j) convert(kept[j], threadIdx.x + j * 64 * WAVES);
        for (uint32_t i = threadIdx.x + kKept * 64 * WAVES; i < eights; i += 64 * WAVES) {
            float x[8];
            read(x, i);
            convert(x, i);
        }
        __syncthreads();
    }
    i32x4 acc[FM] = {};
    for (uint32_t block = first + wave; block < last; block += WAVES * A) {
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const uint32_t at = block + j * WAVES;
            if (at >= last) break;
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                i32x4 lo, hi;
                if constexpr (X == kGiven) {
                    lo = t.a[j][i][0];
                    hi = t.a[j][i][1];
                } else {
                    const uint32_t row = min(16u * i + r16, g.m - 1);
                    const i32x4 *p = reinterpret_cast<const i32x4 *>(lds + row * pitch + at * 128 + 32 * q);
                    lo = p[0];
                    hi = p[1];
                }
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.b[j][0], lo, acc[i], 0, 0, 0);
                acc[i] = __builtin_amdgcn_mfma_i32_16x16x64_i8(t.b[j][1], hi, acc[i], 0, 0, 0);
            }
        }
        if (block + WAVES * A < last) load(block + WAVES * A);
    }
    i32x4 *sums = reinterpret_cast<i32x4 *>(lds);
    if constexpr (X != kGiven) __syncthreads();   // x is read no more
#pragma unroll
    for (int i = 0; i < FM; ++i) sums[(wave * FM + i) * 64 + lane] = acc[i];
    __syncthreads();
    if (wave < FM) {
        i32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[(w * FM + wave) * 64 + lane];
        const uint32_t m = 16 * wave + r16, n = n0 + 4 * q;
        if (m >= g.m || n >= g.n) return;
        if (sp.parts > 1) {
            keep(g, v, part, m, n);
        } else {
            float scale;
            if constexpr (X == kGiven) scale = g.sa[m];
            else scale = RowScale(most[m]).scale;
            finish<OUT>(g, v, scale, m, n);
        }
    }
}

// -------------------------------------------------------------------- join

// The parts' sums; of no parts: k = 0.
template <int OUT>
__global__ __launch_bounds__(256) void join(Int8Args g, uint32_t parts) {
    const uint32_t fours = (g.n + 3) / 4;
    const uint64_t i = static_cast<uint64_t>(block_index()) * 256 + threadIdx.x;
    if (i >= static_cast<uint64_t>(g.m) * fours) return;
    const uint32_t m = static_cast<uint32_t>(i / fours), n = static_cast<uint32_t>(i % fours) * 4;
    const i32x4 *p = reinterpret_cast<const i32x4 *>(g.partial) + i;
    const uint64_t stride = static_cast<uint64_t>(g.m) * fours;
    i32x4 v = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t s = 0; s < parts; ++s) v += p[s * stride];
    finish<OUT>(g, v, g.sa[m], m, n);
}

// ---------------------------------------------------------------- choices

// Bytes of sums of parts where whole tiles fill the card too.
constexpr uint64_t kMostSums = uint64_t(1) << 26;

struct Choice {
    bool large;
    Split split;
};

// What a product takes, in us, by rounds of tiles: a compute unit has one large tile at a time, or two
// small ones, which cover each other's first loads and last stores. Of 24600 products of random sizes, from 33 x
// 64 x 64 to 1.1 TFLOP, the choice takes about 1% longer than the best of ten to sixteen tried (9% or more in one
// of twenty). It is worst where it takes large tiles for 4 to 12 blocks of k, of which it expects too little: 8%
// longer on average, 12267 x 808 x 956 30 us instead of 21.
double tiles_take(uint64_t m, uint64_t n, uint64_t blocks, bool large, uint64_t parts) {
    const uint64_t b = large ? 256 : 128, at_once = large ? kCus : 2 * kCus;
    const uint64_t units = (m + b - 1) / b * ((n + b - 1) / b) * parts;
    const uint64_t rounds = units / at_once, rest = units % at_once;
    const double k = static_cast<double>((blocks + parts - 1) / parts);
    const double start = large ? 11.5 : 4.2, block = large ? 1.28 : 1.14, alone = 0.65;
    double us = static_cast<double>(rounds) * (start + block * k);
    if (large) us += rest != 0 ? start + block * k : 0.0;
    else if (rounds == 0) us += start + (rest <= kCus ? alone : block) * k;
    else if (rest != 0)
        us += (start + block * k) * 0.5 * (1.0 + static_cast<double>(rest) / static_cast<double>(at_once));
    // the parts' sums, written and read
    if (parts > 1) us += 4.0 + static_cast<double>(parts * m * n) * 8 / 5e6;
    return us;
}

Choice choose(uint64_t m, uint64_t n, uint64_t k) {
    Choice c{};
    const uint64_t blocks = (k + 127) / 128, small = (m + 127) / 128 * ((n + 127) / 128);
    uint64_t parts = 1;
    if (small <= kCus / 2) {
        double least = 0.0;
        for (uint64_t q = 1; q <= std::min(kCus / small, blocks); ++q) {
            const uint64_t steps = ((blocks + q - 1) / q + 1) & ~uint64_t(1);
            const double sums = static_cast<double>(q * m * n) * 8 / 5e6 + 0.2 * static_cast<double>(q);
            const double us = 0.5 * static_cast<double>(steps) + (q == 1 ? 0.0 : 4.0 + sums);
            if (q > 1 && us >= least) continue;
            least = us;
            parts = q;
        }
    } else {
        double least = tiles_take(m, n, blocks, false, 1);
        for (uint64_t p = 1; p <= 8 && (p == 1 || (blocks / p >= 8 && p * m * n * 4 <= kMostSums)); ++p)
            for (const bool l : {false, true}) {
                const double us = tiles_take(m, n, blocks, l, p);
                if (us >= least) continue;
                least = us;
                c.large = l;
                parts = p;
            }
    }
    const uint64_t b = c.large ? 256 : 128;
    c.split.tiles_m = static_cast<uint32_t>((m + b - 1) / b);
    c.split.tiles_n = static_cast<uint32_t>((n + b - 1) / b);
    c.split.steps = static_cast<uint32_t>((blocks + parts - 1) / parts);
    if (parts > 1) c.split.steps += c.split.steps & 1;   // blocks go in twos
    c.split.parts = static_cast<uint32_t>((blocks + c.split.steps - 1) / c.split.steps);
    return c;
}

// Few rows: slim reads b once, past LDS, and rows of a for every 16 columns of out. In us, a layer with slim
// and with tiles: 32 x 1000 x 9216 13.6 and 14.6, 64 x 4096 x 4096 15.3 and 16.4, 24 x 4096 x 9216 17.5 and
// 17.4, 64 x 4096 x 9216 27.0 and 19.6, 1 x 25088 x 4096 24.0 and 28.6, 1 x 25088 x 1000 14.2 and 11.7: fitted
// to 104 sizes, of which the rule takes 0.7% longer than the better of both.
constexpr uint64_t kSlimRows = 64;

bool is_slim(uint64_t m, uint64_t n, uint64_t k) {
    const double m1 = static_cast<double>(m), n1 = static_cast<double>(n), k1 = static_cast<double>(k);
    return m <= kSlimRows && n1 * (1.0 + (m1 - 10.0) * k1 / 53000.0) <= 16700.0;
}

// Whether slim converts x itself: a row's bytes in LDS and the padding. Every workgroup converts all of x: in
// us, so and in two launches, 16 x 1000 x 900 6.0 and 6.9, 4 x 4096 x 9216 12.2 and 13.0, 1 x 4096 x 25088 23.1
// and 25.8, 1 x 4096 x 40000 35 and 37, 12 x 4096 x 4096 11.2 and 9.5, 3 x 4096 x 16384 20.4 and 18.8, 24 x 1000
// x 900 8.7 and 8.1.
bool few_bytes(uint64_t m, uint64_t n, uint64_t blocks) {
    return m <= 16 && n <= 8192 && m * (blocks * 128 + 16) <= 45056;
}

// Of slim: where few columns of out leave compute units idle, a long k is split, to a block a wave at
// least.
Split split_slim(uint64_t m, uint64_t n, uint64_t k) {
    Split sp{};
    const uint64_t blocks = (k + 127) / 128;
    sp.tiles_m = 1;
    sp.tiles_n = static_cast<uint32_t>((n + 15) / 16);
    const bool whole = blocks < 64 || (blocks < 128 && few_bytes(m, n, blocks));
    const uint64_t many = std::min<uint64_t>(kCus / sp.tiles_n, blocks / 16);
    const uint64_t parts = whole ? 1 : std::max<uint64_t>(1, many);
    sp.steps = static_cast<uint32_t>((blocks + parts - 1) / parts);
    sp.parts = static_cast<uint32_t>((blocks + sp.steps - 1) / sp.steps);
    return sp;
}

Split split_of(uint64_t m, uint64_t n, uint64_t k) {
    return is_slim(m, n, k) ? split_slim(m, n, k) : choose(m, n, k).split;
}

template <int FM, int OUT, int X>
hipError_t launch_slim(const Int8Args &g, const Split &sp, hipStream_t s) {
    const uint32_t blocks = (g.k + 127) / 128;
    const uint32_t x = X == kGiven ? 0 : g.m * (blocks * 128 + 16);
    constexpr uint32_t kSums = FM * 64 * sizeof(i32x4);   // of a wave
    // sixteen waves keep twice as much of x, too
    const bool long_rows = sp.steps > 64 || sp.parts > 1 || (X != kGiven && g.m * blocks * 16 > kKept * 512);
    dim3 grid;
    if (!grid_of(static_cast<uint64_t>(sp.tiles_n) * sp.parts, long_rows ? 1024 : 512, &grid))
        return hipErrorInvalidConfiguration;
    // Sixteen waves have more of a long row under way, eight leave room for a second workgroup on the
    // compute unit where rows are many and short.
    if (long_rows) slim<FM, OUT, X, 16><<<grid, 1024, std::max(16 * kSums, x), s>>>(g, sp);
    else slim<FM, OUT, X, 8><<<grid, 512, std::max(8 * kSums, x), s>>>(g, sp);
    return hipGetLastError();
}

template <int OUT>
hipError_t launch_join(const Int8Args &g, uint32_t parts, hipStream_t s) {
    dim3 grid;
    if (!grid_of((static_cast<uint64_t>(g.m) * ((g.n + 3) / 4) + 255) / 256, 256, &grid))
        return hipErrorInvalidConfiguration;
    join<OUT><<<grid, 256, 0, s>>>(g, parts);
    return hipGetLastError();
}

template <int OUT>
hipError_t launch(const Int8Args &g, hipStream_t s) {
    if (g.k == 0) return launch_join<OUT>(g, 0, s);
    Split sp;
    hipError_t e;
    if (is_slim(g.m, g.n, g.k)) {
        sp = split_slim(g.m, g.n, g.k);
        if (g.a == nullptr)
            return g.x_bf16 ? launch_slim<1, OUT, PS_BF16>(g, sp, s) : launch_slim<1, OUT, PS_F32>(g, sp, s);
        e = g.m <= 16   ? launch_slim<1, OUT, kGiven>(g, sp, s)
            : g.m <= 32 ? launch_slim<2, OUT, kGiven>(g, sp, s)
                        : launch_slim<4, OUT, kGiven>(g, sp, s);
    } else {
        const Choice c = choose(g.m, g.n, g.k);
        sp = c.split;
        const uint64_t units = static_cast<uint64_t>(sp.tiles_m) * sp.tiles_n * sp.parts;
        if (units > 0xffffffffull / 2) return hipErrorInvalidConfiguration;
        const uint32_t at_once = c.large ? kCus : 2 * kCus, grid = std::min(static_cast<uint32_t>(units), at_once);
        if (sp.parts > 1 && c.large) tiles<4, kSums><<<grid, 256, 0, s>>>(g, sp);
        else if (sp.parts > 1) tiles<2, kSums><<<grid, 256, 0, s>>>(g, sp);
        else if (c.large) tiles<4, OUT><<<grid, 256, 0, s>>>(g, sp);
        else tiles<2, OUT><<<grid, 256, 0, s>>>(g, sp);
        e = hipGetLastError();
    }
    return e != hipSuccess || sp.parts == 1 ? e : launch_join<OUT>(g, sp.parts, s);
}

template <int X, int THREADS>
hipError_t launch_quantize(const Int8QuantArgs &a, dim3 threads, hipStream_t s) {
    dim3 grid;
    if (!grid_of((a.rows + threads.y - 1) / threads.y, THREADS, &grid)) return hipErrorInvalidConfiguration;
    quantize<X, THREADS><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

// As many threads as keep a row, if they are not too many to come and go: in us with 256, 512 and 1024, bf16, 8192 x
// 8192 32, 39 and 99, 4096 x 16384 42, 32 and 49, 4096 x 25088 78, 60 and 61, 128 x 25088 7.7, 5.0 and 4.4, 2048 x
// 100000 201, 165 and 150.
template <int X>
hipError_t launch_quantize(const Int8QuantArgs &a, hipStream_t s) {
    return a.cols <= 512     ? launch_quantize<X, 256>(a, dim3(64, 4), s)
           : a.cols <= 8192  ? launch_quantize<X, 256>(a, dim3(256), s)
           : a.cols <= 32768 ? launch_quantize<X, 512>(a, dim3(512), s)
                             : launch_quantize<X, 1024>(a, dim3(1024), s);
}

}  // namespace

hipError_t launch_quantize_int8(const Int8QuantArgs &a, int dtype, hipStream_t s) {
    return dtype == PS_F32 ? launch_quantize<PS_F32>(a, s) : launch_quantize<PS_BF16>(a, s);
}

size_t int8_workspace(int64_t m, int64_t n, int64_t k) {
    if (m == 0 || n == 0 || k == 0) return 0;
    const uint32_t parts = split_of(m, n, k).parts;
    if (parts == 1) return 0;
    return sizeof(int32_t) * size_t(parts) * size_t(m) * ((size_t(n) + 3) & ~size_t(3));
}

bool int8_converts(int64_t m, int64_t n, int64_t k) {
    return m > 0 && n > 0 && k > 0 && few_bytes(m, n, (k + 127) / 128) && is_slim(m, n, k) &&
           split_slim(m, n, k).parts == 1;
}

hipError_t launch_int8(const Int8Args &g, int out_dtype, hipStream_t s) {
    return out_dtype == PS_F32 ? launch<PS_F32>(g, s) : launch<PS_BF16>(g, s);
}

}  // namespace gadei::learner
