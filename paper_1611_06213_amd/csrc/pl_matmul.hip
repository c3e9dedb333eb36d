// Products of matrices in 8-bit floating point: out = a b^T, a (m x k) and b (n x k) with a
// power-of-two scale per row and block of 128 columns.
//
// Mathematics: out[i, j] = sum over blocks of 2^(ea + eb) * sum over the block's 128
// products, added up in fp32, by one of two instructions:
//
// out in bf16  16 x 16 x 128 on 8-bit operands, which takes the scales of its operands' rows
//              with them (four bytes a row, one per 32 columns; here all four are the block's),
//              so scaling costs no vector work and no second accumulator. It adds products
//              in groups of eight neighbours, of which it keeps 13 bits below the largest
//              (measured, as for the 16 x 16 x 32 form): an error of 2^-19 of the sum of the
//              products' magnitudes, root mean square, far below bf16's 2^-9 of the result
//              unless large products cancel. That is the price of twice the rate.
// out in fp32  16 x 16 x 32 on bf16 operands, at half the rate. An 8-bit value times its block's
//              scale is a bf16 number exactly for scales from 2^-124 on (one conversion instruction
//              for two of them; e4m3's least, 2^-9, is then bf16's least, 2^-133, to which the two
//              smaller scales round), and this instruction's sums are fp32 sums (an error of 2^-27
//              or less, measured).
//
// The first operand is b: then a lane holds four neighbouring columns of out, of one row.
// Lane l gives row l % 16 of either operand, and 32 of the block's columns; which 32 does not
// matter as long as both operands agree, since a block's columns share their scale.
//
// Two kernels: `tiles` stages tiles of both operands in LDS, for many rows of a; `slim`, for
// at most 32 rows of a, reads b, by far the larger operand, straight into registers.
// Where there are too few tiles to fill the card, k is split over workgroups; the parts'
// sums go to the workspace and `join` adds them up in order.
#include <algorithm>

#include "pl_fp8.h"

namespace gadei::learner {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

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

// The same with 32 rows of either operand, of which a lane gives 32 columns of 64.
__device__ __forceinline__ f32x16 mfma(const Operand<false> &b, const Operand<false> &a, f32x16 c) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(b.v, a.v, c, 0, 0, 0, b.scale, 0, a.scale);
}

__device__ __forceinline__ f32x16 mfma(const Operand<true> &b, const Operand<true> &a, f32x16 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
}

__device__ __forceinline__ f32x4 mfma(const Operand<true> &b, const Operand<true> &a, f32x4 c) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b.v[i], a.v[i], c, 0, 0, 0);
    return c;
}

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

__device__ __forceinline__ f32x4 bias_at(const MatmulArgs &g, uint32_t n) {
    return g.bias_bf16 ? load4<PS_BF16>(g.bias, 0, n, g.n) : load4<PS_F32>(g.bias, 0, n, g.n);
}

// What becomes of a sum: four columns from n on of row m.
template <int OUT>
__device__ __forceinline__ void finish(const MatmulArgs &g, f32x4 v, uint32_t m, uint32_t n) {
    const int64_t at = m * g.out_ld + n;
    f32x4 x = v;
    if (g.bias != nullptr) x += bias_at(g, n);
    if (g.relu) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = x[e] < 0.0f ? 0.0f : x[e];   // NaN stays
    }
    if (g.accumulate) x += load4<OUT>(g.out, m * g.out_ld, n, g.n);
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

// 16 bytes of row m's results from column n on; edge: some may lie past the last column.
template <class T>
__device__ __forceinline__ void put(const MatmulArgs &g, u32x4 w, uint32_t m, uint32_t n, bool edge) {
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

// One product, or two in a launch: the workgroups from blocks[0] on are the second's.
struct Products {
    MatmulArgs g[2];
    Split sp[2];
    uint32_t blocks[2], join_blocks[2];
};

// ------------------------------------------------------------------- tiles

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

// Tiles of 64 FM x 64 FN by 2 x 2 waves, each FM x FN instructions of 32 x 32.
//
// Bound by the matrix pipes and, at large sizes, by power: the clock falls from 2.4 to 1.75 GHz,
// and the same product of zeros takes three quarters of the time. 8192^3 to bf16 takes 424 to 510
// us (2.2 to 2.6 PFLOP/s), 16384 x 4096 x 4096 230 (2.4), and to fp32, by bf16 instructions, 450
// to 500 (1.1 to 1.2). A step of 256 x 256 tiles reads half of what four 128 x 128 tiles read from LDS (8192^3
// takes 606 us with those), and 256 x 128, for fp32 results, leaves registers for the operands in
// bf16.
//
// A step is half a block, 64 columns. LDS holds four steps of either operand, which copies bring
// there from memory without registers; the registers hold the step that multiplies and the
// one after it. So in step s, step s + 1 is read from LDS, step s + 4 is copied to where s was,
// and the copies have three steps to arrive: at the end of a step only those of the one
// before the last are waited for.
template <int FM, int FN, int OUT>
__device__ __forceinline__ void take_units(const MatmulArgs &g, const Split &sp, uint32_t unit,
                                           uint32_t stride, uint8_t *a0, uint8_t *a1, uint8_t *a2,
                                           uint8_t *a3, uint8_t *b0, uint8_t *b1, uint8_t *b2,
                                           uint8_t *b3, float *bias) {
    constexpr int BM = 64 * FM, BN = 64 * FN;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const int wm = wave % 2 * (32 * FM), wn = wave / 2 * (32 * FN);
    const int q = lane >> 5, r32 = lane & 31;

    // A copy takes 16 rows of 64 bytes. Rows past the matrix are outside the buffers' bounds and
    // read as zeros, as are their scales. 16 bytes c of row r lie at 64 r + 16 (c ^ (r / 4 % 4)),
    // so that the 16 lanes that LDS serves at once (of rows 0-3, 12-15, 20-23 and 24-27, or of
    // the other 16) lie in different banks.
    const uint32_t from = (lane >> 2) * ld + (((lane & 3) ^ ((lane >> 4) & 3)) << 4);
    const int low = r32 * 64 + (((2 * q) ^ (r32 >> 2 & 3)) << 4);
    const int high = r32 * 64 + (((2 * q + 1) ^ (r32 >> 2 & 3)) << 4);

    // a work unit: a tile and a part of k
    uint32_t m0, n0, part, first, last;
    Buffer rows_a, rows_b;
    auto take = [&](uint32_t unit) {
        uint32_t tile_m, tile_n;
        place(sp, unit, &tile_m, &tile_n, &part);
        m0 = tile_m * BM;
        n0 = tile_n * BN;
        first = part * sp.steps;
        last = min(blocks, first + sp.steps);   // first < last, as the host splits
        rows_a = Buffer(g.a + static_cast<uint64_t>(m0) * ld, min(g.m - m0, uint32_t(BM)) * ld);
        rows_b = Buffer(g.b + static_cast<uint64_t>(n0) * ld, min(g.n - n0, uint32_t(BN)) * ld);
    };
    // The wave's copies of a step (of block `block`, half 0 or 1): FM of a, FN of b. Blocks past the
    // last: no bytes.
    auto copy = [&](uint8_t *a, uint8_t *b, int i, uint32_t block, int half) {
        const uint32_t lanes = block < last ? from : Buffer::kOutside;
        if (i < FM)
            rows_a.to_lds(a + (wave * FM + i) * 1024, lanes,
                          (wave * FM + i) * 16 * ld + block * 128 + half * 64);
        else
            rows_b.to_lds(b + (wave * FN + i - FM) * 1024, lanes,
                          (wave * FN + i - FM) * 16 * ld + block * 128 + half * 64);
    };

    // The scales of four blocks are a word of each row. These are shifted so that the byte of the
    // step that is being read is the lowest; the next words are loaded a block
    // ahead.
    uint32_t sa[FM], sb[FN], next_a[FM], next_b[FN];
    auto load_words = [&](uint32_t (&a)[FM], uint32_t (&b)[FN], uint32_t block, bool wanted) {
        const uint64_t group = min(block, blocks - 1) >> 2;
        const Buffer ga(g.sa + group * g.m, g.m * 4), gb(g.sb + group * g.n, g.n * 4);
        const uint32_t la = wanted ? (m0 + wm + r32) * 4 : Buffer::kOutside;
        const uint32_t lb = wanted ? (n0 + wn + r32) * 4 : Buffer::kOutside;
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = ga.word(la + 128 * i);
#pragma unroll
        for (int j = 0; j < FN; ++j) b[j] = gb.word(lb + 128 * j);
    };
    // The bias of the thread's column of the tile, zero where there is none; asked for before a unit's
    // copies, kept in LDS for its end.
    const Buffer bias32(g.bias, g.bias != nullptr && !g.bias_bf16 ? g.n * 4 : 0);
    const Buffer bias16(g.bias, g.bias != nullptr && g.bias_bf16 ? g.n * 2 : 0);
    uint32_t bias_word, bias_half;
    auto column_bias = [&] { return __uint_as_float(bias_word | bias_half << 16); };
    // The first four steps' copies and the first words. After step 1's come two steps' copies and
    // one load of words, as after every step's in the loop: its waits count on that.
    auto begin = [&] {
        bias_word = bias32.word((n0 + threadIdx.x) * 4);
        bias_half = bias16.half((n0 + threadIdx.x) * 2);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) copy(a0, b0, i, first, 0);
        load_words(sa, sb, first, true);
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) copy(a1, b1, i, first, 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) copy(a2, b2, i, first + 1, 0);
        __builtin_amdgcn_sched_barrier(0);
        load_words(next_a, next_b, first + 1, ((first + 1) & 3) == 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < FM + FN; ++i) copy(a3, b3, i, first + 1, 1);
        __builtin_amdgcn_sched_barrier(0);
    };

    using Op = Operand<OUT == PS_F32>;
    struct Raw { i32x4 lo, hi; };
    struct Step { Raw a[FM], b[FN]; uint32_t sa[FM], sb[FN]; };
    f32x16 acc[FM][FN];
    auto read_a = [&](Step &s, const uint8_t *at, int i) {
        const uint8_t *p = at + (wm + 32 * i) * 64;
        s.a[i] = Raw{*reinterpret_cast<const i32x4 *>(p + low), *reinterpret_cast<const i32x4 *>(p + high)};
        s.sa[i] = sa[i];
    };
    auto read_b = [&](Step &s, const uint8_t *at, int j) {
        const uint8_t *p = at + (wn + 32 * j) * 64;
        s.b[j] = Raw{*reinterpret_cast<const i32x4 *>(p + low), *reinterpret_cast<const i32x4 *>(p + high)};
        s.sb[j] = sb[j];
    };
    // Multiply `now`, read `next` (from a and b), copy half `half` of block `block` to a_to and b_to.
    auto step = [&](const Step &now, Step &next, const uint8_t *a, const uint8_t *b, uint8_t *a_to,
                    uint8_t *b_to, uint32_t block, int half) {
        // Reads and copies one at a time between the products: the memory pipeline takes a copy every
        // 16 cycles from four waves, and a wave that has to wait there issues no products. The reads
        // end early, so that none is waited for at the step's end.
        constexpr int N = FM + FN, S = FM * FN;
        Op fa, fb[FN];
#pragma unroll
        for (int t = 0; t < S; ++t) {
            const int i = t / FN, j = t % FN;
            if (j == 0) fa.set(now.a[i].lo, now.a[i].hi, now.sa[i]);
            if (i == 0) fb[j].set(now.b[j].lo, now.b[j].hi, now.sb[j]);
            acc[i][j] = mfma(fb[j], fa, acc[i][j]);
#pragma unroll
            for (int c = t * 3 * N / (2 * S); c < (t + 1) * 3 * N / (2 * S) && c < N; ++c) {
                if (c < FM) read_a(next, a, c);
                else read_b(next, b, c - FM);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = (t * N + N / 2) / S; c < ((t + 1) * N + N / 2) / S && c < N; ++c)
                copy(a_to, b_to, c, block, half);
            __builtin_amdgcn_sched_barrier(0);
        }
        // This wave's copies but those of the last two steps have arrived, and its reads; then
        // everyone's. Since those copies it has issued 2 (FM + FN) more and the loads of one
        // block's words.
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(3 * (FM + FN)) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    Step x, y;
    // A block's second step reads the next block's first half, and so takes that block's words;
    // the words of the block after it are loaded then, if they are of another group. There
    // is no branch in a step: the compiler would move products across it.
    auto block = [&](uint32_t k, uint8_t *pa0, uint8_t *pb0, uint8_t *pa1, uint8_t *pb1, uint8_t *pa2,
                     uint8_t *pb2) {
        step(x, y, pa1, pb1, pa0, pb0, k + 2, 0);
        const bool group = ((k + 1) & 3) == 0;
        const uint32_t keep = k + 1 < last ? 0xffffffffu : 0;   // a block of zeros: any finite scale
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = (group ? next_a[i] : sa[i] >> 8) & keep;
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] = (group ? next_b[j] : sb[j] >> 8) & keep;
        load_words(next_a, next_b, k + 2, ((k + 2) & 3) == 0);
        __builtin_amdgcn_sched_barrier(0);
        step(y, x, pa2, pb2, pa1, pb1, k + 2, 1);
    };

    asm volatile("; the first unit's copies");
    take(unit);
    begin();
    for (;;) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f32x16{};
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(3 * (FM + FN)) : "memory");   // steps 0 and 1
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] >>= 8 * (first & 3);
#pragma unroll
        for (int j = 0; j < FN; ++j) sb[j] >>= 8 * (first & 3);
#pragma unroll
        for (int i = 0; i < FM; ++i) read_a(x, a0, i);
#pragma unroll
        for (int j = 0; j < FN; ++j) read_b(x, b0, j);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();   // a0 and b0 may be written
        asm volatile("" ::: "memory");
        // an odd number of blocks is followed by one of zeros: a loop with a way out in its middle
        // would have the compiler move all sums from register to register
        for (uint32_t k = first; k < last; k += 2) {
            block(k, a0, b0, a1, b1, a2, b2);
            block(k + 1, a2, b2, a3, b3, a0, b0);
        }

        // The results go out from the registers, while the next unit's first copies are under way.
        // The lane's number is hidden from the compiler here: it would compute all addresses below
        // before the loop, and have no registers for them in it.
        uint32_t lane1 = threadIdx.x & 63;
        asm volatile("" : "+v"(lane1));
        const uint32_t q1 = lane1 >> 5, r1 = lane1 & 31, hi1 = lane1 >> 4 & 1;
        const uint32_t m1 = m0 + wm, n1 = n0 + wn, part1 = part;
        const bool edge = n0 + BN > g.n, sums = sp.parts > 1, with_bias = g.bias != nullptr && !sums;
        unit += stride;
        const bool more = unit < sp.tiles_m * sp.tiles_n * sp.parts;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // the last copies write zeros to LDS
        if (threadIdx.x < BN) bias[threadIdx.x] = column_bias();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (more && !g.accumulate) {
            take(unit);
            begin();
        }
        f32x4 old[2][4] = {};   // what out holds
#pragma unroll
        for (int j0 = 0; j0 < FN; j0 += 2) {   // 64 columns of a row after one another: a line of bf16
#pragma unroll
            for (int ij = 0; ij < 2 * FM; ++ij) {
                const int i = ij / 2, j = j0 + ij % 2;
                const uint32_t m = m1 + 32 * i + r1;
                if (g.accumulate && !sums && ij % 2 == 0 && m < g.m) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        old[e / 4][e % 4] =
                            load4<OUT>(g.out, m * g.out_ld, n1 + 32 * j0 + 8 * e + 4 * q1, g.n);
                }
                f32x4 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    // a lane holds row r1's columns 8 e + 4 q1 + 0..3 of each 32
                    v[e] = f32x4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2],
                                 acc[i][j][4 * e + 3]};
                    if (with_bias)
                        v[e] += *reinterpret_cast<const f32x4 *>(bias + wn + 32 * j + 8 * e + 4 * q1);
                    if (g.relu && !sums) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[e][c] = v[e][c] < 0.0f ? 0.0f : v[e][c];   // NaN stays
                    }
                    if (g.accumulate && !sums) v[e] += old[j - j0][e];
                }
                // Lanes exchange so that a store writes 64 neighbouring bytes of each of 16 rows: with 32
                // bytes of 32 rows, results past the caches were written to memory 1.7 times.
                if (OUT == PS_F32 || sums) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        u32x4 w[2] = {__builtin_bit_cast(u32x4, v[2 * h]),
                                      __builtin_bit_cast(u32x4, v[2 * h + 1])};
                        swap_rows(w[0], w[1]);
                        const uint32_t n = n1 + 32 * j + 16 * h + 8 * hi1 + 4 * q1;
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const uint32_t to = m1 + 32 * i + 16 * t + (lane1 & 15);
                            if (to < g.m && sums) {
                                if (n < g.n) keep(g, __builtin_bit_cast(f32x4, w[t]), part1, to, n);
                            } else if (to < g.m) {
                                put<float>(g, w[t], to, n, edge);
                            }
                        }
                    }
                } else {
                    // 16 bytes of bf16 first: the halves of the wave exchange fours
                    u32x4 w[2];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const auto p = __builtin_amdgcn_permlane32_swap(
                                bf16x2_rne(v[2 * h][2 * c], v[2 * h][2 * c + 1]),
                                bf16x2_rne(v[2 * h + 1][2 * c], v[2 * h + 1][2 * c + 1]), false, false);
                            w[h][c] = p[0];
                            w[h][2 + c] = p[1];
                        }
                    swap_rows(w[0], w[1]);
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const uint32_t to = m1 + 32 * i + 16 * t + (lane1 & 15);
                        if (to < g.m) put<uint16_t>(g, w[t], to, n1 + 32 * j + 16 * hi1 + 8 * q1, edge);
                    }
                }
            }
        }
        if (more && g.accumulate) {
            take(unit);
            begin();
        }
        if (!more) break;
    }
}

// Small products leave most compute units idle, or wait for their first bytes most of the time. A
// layer's two backward products in one launch take, in fp32, quantisation and joining included, 16.5 us
// instead of 23.0 for 57 x 1000 x 900, 18.6 instead of 27.4 for 300 x 1000 x 1000, 35 instead of 45
// for 1000 x 2000 x 2000.
template <int FM, int FN, int OUT0, int OUT1>
__global__ __launch_bounds__(256, FM == 2 ? 2 : 1) void tiles(Products both) {
    constexpr int A = 64 * FM * 64, B = 64 * FN * 64;
    // buffers that the compiler can tell apart: it would wait for all copies before every
    // read of LDS if it could not
    __shared__ __attribute__((aligned(128))) uint8_t a0[A], a1[A], a2[A], a3[A], b0[B], b1[B], b2[B], b3[B];
    __shared__ __attribute__((aligned(16))) float bias[64 * FN];
    const bool second = blockIdx.x >= both.blocks[0];
    const uint32_t unit = blockIdx.x - (second ? both.blocks[0] : 0), stride = both.blocks[second];
    if (OUT0 == OUT1 || !second)
        take_units<FM, FN, OUT0>(both.g[second], both.sp[second], unit, stride, a0, a1, a2, a3, b0, b1, b2,
                                 b3, bias);
    else
        take_units<FM, FN, OUT1>(both.g[1], both.sp[1], unit, stride, a0, a1, a2, a3, b0, b1, b2, b3,
                                   bias);
}

// -------------------------------------------------------------------- slim

// 16 rows of b (columns of out) a workgroup and up to 16 FM rows of a: bound by reading b, once,
// straight into registers. The waves take the blocks of k in turn, the loads of several blocks under
// way in each, and add up their sums in LDS, in order: no part of k goes through memory. 1 x 4096 x
// 25088 takes 20 us (5.1 TB/s of b).
//
// X >= 0: a is not in 8-bit form yet but given as x. Every workgroup converts all of it, into LDS,
// while its first rows of b are under way: for few rows that is less than a launch.
constexpr int kGiven = -1;
template <int FM>
constexpr int kAhead = FM == 1 ? 4 : 2;   // blocks whose loads are issued together

template <int FM, int OUT, int X, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void slim(MatmulArgs g, Split sp) {
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    constexpr int A = kAhead<FM>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int q = lane >> 4, r16 = lane & 15;
    const uint32_t part = block_index() / sp.tiles_n, n0 = block_index() % sp.tiles_n * 16;
    if (part >= sp.parts) return;
    const uint32_t blocks = (g.k + 127) / 128, ld = blocks * 128;
    const uint32_t first = part * sp.steps, last = min(blocks, first + sp.steps);
    const uint32_t pitch = ld + 16;   // of x's rows in LDS: in different banks
    uint8_t *const bytes = lds + g.m * pitch;   // x's scales: `blocks` of a row
    // rows past a matrix, and blocks past the last, read as zeros
    const Buffer rows_b(g.b + static_cast<uint64_t>(n0) * ld, min(g.n - n0, 16u) * ld);
    const Buffer rows_a(g.a, g.m * ld);
    const uint32_t from = r16 * ld + 32 * q;

    struct Ahead {
        i32x4 b[A][2], a[A][FM][2];
        uint32_t sb[A], sa[A][FM];
    } t;
    auto load = [&](uint32_t block) {
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const uint32_t at = block + j * WAVES;
            const bool in = at < last;
            const uint32_t lanes = in ? from : Buffer::kOutside;
            t.b[j][0] = rows_b.sixteen(lanes, at * 128);
            t.b[j][1] = rows_b.sixteen(lanes, at * 128 + 16);
            const uint32_t group = in ? at >> 2 : 0;
            t.sb[j] = Buffer(g.sb + static_cast<uint64_t>(group) * g.n, g.n * 4).word((n0 + r16) * 4);
            if constexpr (X == kGiven) {
                const Buffer words(g.sa + static_cast<uint64_t>(group) * g.m, g.m * 4);
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    t.a[j][i][0] = rows_a.sixteen(lanes, 16 * i * ld + at * 128);
                    t.a[j][i][1] = rows_a.sixteen(lanes, 16 * i * ld + at * 128 + 16);
                    t.sa[j][i] = words.word((16 * i + r16) * 4);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // all under way before the first is used
    };
    load(first + wave);
    if constexpr (X != kGiven) {
        constexpr int kTogether = 4;
        const uint32_t group = threadIdx.x >> 4, e = threadIdx.x & 15;   // sixteen lanes a block
        for (uint32_t i0 = group; i0 < g.m * blocks; i0 += kTogether * 4 * WAVES) {
            Bits8<X> x[kTogether];
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const uint32_t i = i0 + j * 4 * WAVES, m = i / blocks, col = i % blocks * 128 + 8 * e;
                const int count = m >= g.m || col >= g.k ? 0 : static_cast<int>(min(g.k - col, 8u));
                const int64_t at = m * g.x_ld + col;
                if (count == 8) x[j] = load8<X>(g.x, at);
                else x[j] = load8_some<X>(g.x, at, count);
            }
#pragma unroll
            for (int j = 0; j < kTogether; ++j) {
                const uint32_t i = i0 + j * 4 * WAVES, m = i / blocks, col = i % blocks * 128 + 8 * e;
                const uint32_t byte = scale_byte(most_of_block(most8<X>(x[j])));
                if (m >= g.m) break;
                *reinterpret_cast<u32x2 *>(lds + m * pitch + col) =
                    u32x2{four(x[j], 0, as_scale(byte)), four(x[j], 1, as_scale(byte))};
                if (e == 0) bytes[i] = static_cast<uint8_t>(byte);
            }
        }
        __syncthreads();
    }
    const uint32_t rx = min(uint32_t(r16), g.m - 1);
    f32x4 acc[FM] = {};
    for (uint32_t block = first + wave; block < last; block += WAVES * A) {
#pragma unroll
        for (int j = 0; j < A; ++j) {
            const uint32_t at = block + j * WAVES;
            if (at >= last) break;
            Operand<OUT == PS_F32> fb, fa;
            fb.set(t.b[j][0], t.b[j][1], t.sb[j] >> (8 * (at & 3)));
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if constexpr (X == kGiven) {
                    fa.set(t.a[j][i][0], t.a[j][i][1], t.sa[j][i] >> (8 * (at & 3)));
                } else {
                    const i32x4 *p = reinterpret_cast<const i32x4 *>(lds + rx * pitch + at * 128 + 32 * q);
                    fa.set(p[0], p[1], bytes[rx * blocks + at]);
                }
                acc[i] = mfma(fb, fa, acc[i]);
            }
        }
        if (block + WAVES * A < last) load(block + WAVES * A);
    }
    f32x4 *sums = reinterpret_cast<f32x4 *>(lds);
    if constexpr (X != kGiven) __syncthreads();   // x is read no more
#pragma unroll
    for (int i = 0; i < FM; ++i) sums[(wave * FM + i) * 64 + lane] = acc[i];
    __syncthreads();
    if (wave < FM) {
        f32x4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[(w * FM + wave) * 64 + lane];
        const uint32_t m = 16 * wave + r16, n = n0 + 4 * q;
        if (m >= g.m || n >= g.n) return;
        if (sp.parts > 1) keep(g, v, part, m, n);
        else finish<OUT>(g, v, m, n);
    }
}

// -------------------------------------------------------------------- join

// The parts' sums, in their order.
template <int OUT0, int OUT1>
__global__ __launch_bounds__(256) void join(Products both) {
    const bool second = blockIdx.x >= both.join_blocks[0];
    const MatmulArgs &g = both.g[second];
    const uint32_t fours = (g.n + 3) / 4, parts = both.sp[second].parts;
    const uint32_t block = blockIdx.x - (second ? both.join_blocks[0] : 0);
    const uint64_t i = static_cast<uint64_t>(block) * 256 + threadIdx.x;
    if (i >= static_cast<uint64_t>(g.m) * fours) return;
    const uint32_t m = static_cast<uint32_t>(i / fours), n = static_cast<uint32_t>(i % fours) * 4;
    const f32x4 *p = reinterpret_cast<const f32x4 *>(g.partial) + i;
    const uint64_t stride = static_cast<uint64_t>(g.m) * fours;
    f32x4 v = {0, 0, 0, 0};
#pragma unroll 8
    for (uint32_t s = 0; s < parts; ++s) v += p[s * stride];
    if (OUT0 == OUT1 || !second) finish<OUT0>(g, v, m, n);
    else finish<OUT1>(g, v, m, n);
}

// k = 0: sums of no terms.
template <int OUT>
__global__ __launch_bounds__(256) void empty(MatmulArgs g) {
    const uint32_t fours = (g.n + 3) / 4;
    const uint64_t i = static_cast<uint64_t>(block_index()) * 256 + threadIdx.x;
    if (i >= static_cast<uint64_t>(g.m) * fours) return;
    finish<OUT>(g, f32x4{0, 0, 0, 0}, static_cast<uint32_t>(i / fours),
                static_cast<uint32_t>(i % fours) * 4);
}

// ---------------------------------------------------------------- choices

// In us, with slim and with tiles: 32 x 4096 x 9216 16.0 and 14.4, 64 x 4096 x 9216 24.7 and 16.4.
constexpr uint32_t kSlimRows = 32;

// Bytes of sums of parts where whole tiles fill the card too.
constexpr uint64_t kMostSums = uint64_t(1) << 26;

struct Choice {
    int bm, bn;
    Split split;
};

// What a product takes, in us, by rounds of tiles: a compute unit has one large tile at a time, or
// two small ones, which cover each other's first loads and last stores; the last ones of many take
// less, as some have a compute unit each. Fitted to 170 products of random sizes from 512 x 512 x
// 64 to 16384 x 25088 x 16384.
double tiles_take(uint64_t m, uint64_t n, uint64_t blocks, bool wide, bool large, uint64_t parts) {
    const uint64_t bm = large ? 256 : 128, bn = large && !wide ? 256 : 128;
    const uint64_t units = (m + bm - 1) / bm * ((n + bn - 1) / bn) * parts, at_once = large ? kCus : 2 * kCus;
    const uint64_t rounds = units / at_once, rest = units % at_once;
    const double k = static_cast<double>((blocks + parts - 1) / parts);
    const double start = large ? (wide ? 8.0 : 11.5) : wide ? 6.8 : 4.2;
    const double block = large ? (wide ? 1.5 : 1.28) : wide ? 1.57 : 1.14, alone = wide ? 0.91 : 0.65;
    double us = static_cast<double>(rounds) * (start + block * k);
    if (large) us += rest != 0 ? start + block * k : 0.0;
    else if (rounds == 0) us += start + (rest <= kCus ? alone : block) * k;
    else if (rest != 0)
        us += (start + block * k) * 0.5 * (1.0 + static_cast<double>(rest) / static_cast<double>(at_once));
    // the parts' sums, written and read
    if (parts > 1) us += 4.0 + static_cast<double>(parts * m * n) * 8 / 5e6;
    return us;
}

// For more than kSlimRows rows of a.
Choice choose(uint64_t m, uint64_t n, uint64_t k, bool wide) {
    Choice c{};
    const uint64_t blocks = (k + 127) / 128, small = (m + 127) / 128 * ((n + 127) / 128);
    bool large = false;
    uint64_t parts = 1;
    if (small <= kCus / 2) {
        // Parts of k until every compute unit has a workgroup, unless the joining takes longer: in us,
        // 64 x 128 x 4096 10.6 in parts of eight blocks and 8.8 of four, 57 x 900 x 1000 to bf16 8.9 in
        // parts of four and 8.6 whole (with the other backward product and their joining 14.3 and 13.8),
        // to fp32 10.3 in parts of two and 12.9 whole.
        double least = 0.0;
        for (uint64_t q = 1; q <= std::min(kCus / small, blocks); ++q) {
            const uint64_t steps = ((blocks + q - 1) / q + 1) & ~uint64_t(1);
            const double sums = static_cast<double>(q * m * n) * 8 / 5e6 + 0.2 * static_cast<double>(q);
            const double join = q == 1 ? 0.0 : 4.0 + sums;
            const double us = (wide ? 0.9 : 0.5) * static_cast<double>(steps) + join;
            if (q > 1 && us >= least) continue;
            least = us;
            parts = q;
        }
    } else {
        // Large tiles read LDS and the caches least, small ones lose less where tiles are few or k
        // is short; parts fill the last round (1280 x 4096 x 22272 196 us whole and 111 in parts,
        // 256 x 21248 x 24320 304 and 163). Over the fitted sizes, large tiles wherever there are
        // 256 of them took 9% longer than the better of both (15% to fp32), this rule 0.6%.
        double least = tiles_take(m, n, blocks, wide, false, 1);
        for (uint64_t p = 1; p <= 8 && (p == 1 || (blocks / p >= 8 && p * m * n * 4 <= kMostSums)); ++p)
            for (const bool l : {false, true}) {
                const double us = tiles_take(m, n, blocks, wide, l, p);
                if (us >= least) continue;
                least = us;
                large = l;
                parts = p;
            }
    }
    c.bm = large ? 256 : 128;
    c.bn = large && !wide ? 256 : 128;
    c.split.tiles_m = static_cast<uint32_t>((m + c.bm - 1) / c.bm);
    c.split.tiles_n = static_cast<uint32_t>((n + c.bn - 1) / c.bn);
    c.split.steps = static_cast<uint32_t>((blocks + parts - 1) / parts);
    if (parts > 1) c.split.steps += c.split.steps & 1;   // blocks go in twos
    c.split.parts = static_cast<uint32_t>((blocks + c.split.steps - 1) / c.split.steps);
    return c;
}

// Whether slim converts x itself: a row's bytes in LDS, its scales and the padding. Every workgroup
// converts all of x: 1 x 4096 (4 KB) takes 6.0 us, 7.6 in two launches, 2 x 25088 (50 KB) 22.7 and
// 22.6, but 16 x 4096 (66 KB) 11.6 and 9.2, all with 4096 columns of out.
bool few_bytes(uint64_t m, uint64_t blocks) { return m <= 16 && m * (blocks * 129 + 16) <= 51200; }

// Of slim: where few columns of out leave compute units idle, a long k is split, to a block a wave
// at least. In us, whole and split, joining included: 3 x 300 x 24000 17.8 and 8.3, 32 x 1000 x
// 8192 13.5 and 9.4, 3 x 1000 x 8192 7.9 and 8.3, 32 x 300 x 4096 8.2 and 8.6. A split product's x
// is converted first, which for few bytes pays from 128 blocks on (1 x 70 x 17000 with its
// conversion 12.0 and 9.7, 1 x 70 x 8192 7.6 and 10.2).
Split split_slim(uint64_t m, uint64_t n, uint64_t k) {
    Split sp{};
    const uint64_t blocks = (k + 127) / 128;
    sp.tiles_m = 1;
    sp.tiles_n = static_cast<uint32_t>((n + 15) / 16);
    const bool whole = blocks < 64 || (blocks < 128 && few_bytes(m, blocks));
    const uint64_t many = std::min<uint64_t>(kCus / sp.tiles_n, blocks / 16);
    const uint64_t parts = whole ? 1 : std::max<uint64_t>(1, many);
    sp.steps = static_cast<uint32_t>((blocks + parts - 1) / parts);
    sp.parts = static_cast<uint32_t>((blocks + sp.steps - 1) / sp.steps);
    return sp;
}

template <int FM, int OUT, int X>
hipError_t launch_slim(const MatmulArgs &g, const Split &sp, hipStream_t s) {
    const uint32_t blocks = (g.k + 127) / 128;
    const uint32_t x = X == kGiven ? 0 : g.m * (blocks * 128 + 16) + g.m * blocks;
    constexpr uint32_t kSums = FM * 64 * sizeof(f32x4);   // of a wave
    const bool long_rows = sp.steps > 64 || sp.parts > 1;
    dim3 grid;
    if (!grid_of(static_cast<uint64_t>(sp.tiles_n) * sp.parts, long_rows ? 1024 : 512, &grid))
        return hipErrorInvalidConfiguration;
    // Sixteen waves have more of a long row under way, eight leave room for a second workgroup on
    // the compute unit where rows are many and short: a layer of 1 x 4096 x 25088 20.6 us with 16, 23.3
    // with 8; 1 x 25088 x 4096 32.3 and 22.3.
    if (long_rows) slim<FM, OUT, X, 16><<<grid, 1024, std::max(16 * kSums, x), s>>>(g, sp);
    else slim<FM, OUT, X, 8><<<grid, 512, std::max(8 * kSums, x), s>>>(g, sp);
    return hipGetLastError();
}

uint64_t join_blocks(const MatmulArgs &g) {
    return (static_cast<uint64_t>(g.m) * ((g.n + 3) / 4) + 255) / 256;
}

// The product's work units; at most `most` workgroups take them.
bool place_product(const MatmulArgs &g, const Choice &c, uint32_t most, int i, Products *p) {
    const uint64_t units = static_cast<uint64_t>(c.split.tiles_m) * c.split.tiles_n * c.split.parts;
    const uint64_t joins = c.split.parts > 1 ? join_blocks(g) : 0;
    if (units > 0xffffffffull / 2 || joins > 0xffffffffull / 512) return false;
    p->g[i] = g;
    p->sp[i] = c.split;
    p->blocks[i] = std::min(static_cast<uint32_t>(units), most);
    p->join_blocks[i] = static_cast<uint32_t>(joins);
    return true;
}

template <int OUT0, int OUT1>
hipError_t launch_join(const Products &p, hipStream_t s) {
    const hipError_t e = hipGetLastError();
    const uint32_t joins = p.join_blocks[0] + p.join_blocks[1];
    if (e != hipSuccess || joins == 0) return e;
    join<OUT0, OUT1><<<joins, 256, 0, s>>>(p);
    return hipGetLastError();
}

template <int OUT>
hipError_t launch(const MatmulArgs &g, hipStream_t s) {
    if (g.k == 0) {
        dim3 grid;
        if (!grid_of(join_blocks(g), 256, &grid)) return hipErrorInvalidConfiguration;
        empty<OUT><<<grid, 256, 0, s>>>(g);
        return hipGetLastError();
    }
    Products p{};
    if (g.m <= kSlimRows) {
        Choice c{};
        c.split = split_slim(g.m, g.n, g.k);
        if (!place_product(g, c, 0, 0, &p)) return hipErrorInvalidConfiguration;
        const hipError_t e = g.m <= 16 ? launch_slim<1, OUT, kGiven>(g, c.split, s)
                                       : launch_slim<2, OUT, kGiven>(g, c.split, s);
        return e != hipSuccess ? e : launch_join<OUT, OUT>(p, s);
    }
    const Choice c = choose(g.m, g.n, g.k, OUT == PS_F32);
    if (!place_product(g, c, c.bm == 128 ? 2 * kCus : kCus, 0, &p)) return hipErrorInvalidConfiguration;
    if (c.bm == 128) tiles<2, 2, OUT, OUT><<<p.blocks[0], 256, 0, s>>>(p);
    else tiles<4, OUT == PS_F32 ? 2 : 4, OUT, OUT><<<p.blocks[0], 256, 0, s>>>(p);
    return launch_join<OUT, OUT>(p, s);
}

template <int OUT0, int OUT1>
hipError_t launch_two(const MatmulArgs &a, const MatmulArgs &b, hipStream_t s) {
    Products p{};
    if (!place_product(a, choose(a.m, a.n, a.k, OUT0 == PS_F32), kCus, 0, &p) ||
        !place_product(b, choose(b.m, b.n, b.k, OUT1 == PS_F32), kCus, 1, &p))
        return hipErrorInvalidConfiguration;
    tiles<2, 2, OUT0, OUT1><<<p.blocks[0] + p.blocks[1], 256, 0, s>>>(p);
    return launch_join<OUT0, OUT1>(p, s);
}

bool is_small(const MatmulArgs &g, int out_dtype) {
    if (g.m <= kSlimRows || g.n == 0 || g.k == 0) return false;
    const Choice c = choose(g.m, g.n, g.k, out_dtype == PS_F32);
    return c.bm == 128 && static_cast<uint64_t>(c.split.tiles_m) * c.split.tiles_n * c.split.parts <= kCus;
}

}  // namespace

size_t matmul_workspace(int64_t m, int64_t n, int64_t k, int out_dtype) {
    if (m == 0 || n == 0 || k == 0) return 0;
    const Split split = m <= kSlimRows ? split_slim(m, n, k) : choose(m, n, k, out_dtype == PS_F32).split;
    const uint32_t parts = split.parts;
    if (parts == 1) return 0;
    return sizeof(float) * size_t(parts) * size_t(m) * ((size_t(n) + 3) & ~size_t(3));
}

bool converts(int64_t m, int64_t n, int64_t k) {
    return m > 0 && n > 0 && k > 0 && few_bytes(m, (k + 127) / 128) && split_slim(m, n, k).parts == 1;
}

hipError_t launch_matmul(const MatmulArgs &a, int out_dtype, hipStream_t s) {
    return out_dtype == PS_F32 ? launch<PS_F32>(a, s) : launch<PS_BF16>(a, s);
}

bool pairs(const MatmulArgs &a, int a_dtype, const MatmulArgs &b, int b_dtype) {
    return is_small(a, a_dtype) && is_small(b, b_dtype);
}

hipError_t launch_matmul_two(const MatmulArgs &a, int a_dtype, const MatmulArgs &b, int b_dtype,
                             hipStream_t s) {
    if (a_dtype != b_dtype)
        return a_dtype == PS_BF16 ? launch_two<PS_BF16, PS_F32>(a, b, s)
                                  : launch_two<PS_BF16, PS_F32>(b, a, s);
    return a_dtype == PS_F32 ? launch_two<PS_F32, PS_F32>(a, b, s) : launch_two<PS_BF16, PS_BF16>(a, b, s);
}

hipError_t launch_convert_matmul(const MatmulArgs &a, int x_dtype, int out_dtype, hipStream_t s) {
    Split whole{1, (a.n + 15) / 16, 1, (a.k + 127) / 128};
    if (out_dtype == PS_F32)
        return x_dtype == PS_F32 ? launch_slim<1, PS_F32, PS_F32>(a, whole, s)
                                 : launch_slim<1, PS_F32, PS_BF16>(a, whole, s);
    return x_dtype == PS_F32 ? launch_slim<1, PS_BF16, PS_F32>(a, whole, s)
                             : launch_slim<1, PS_BF16, PS_BF16>(a, whole, s);
}

}  // namespace gadei::learner
