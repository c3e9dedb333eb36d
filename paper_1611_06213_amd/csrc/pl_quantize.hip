// Matrices to 8-bit floating point with a power-of-two scale per block of 128.
//
// The numbers are those of pl_fp8.h.
//
// Bound by memory: x is read once and one byte per element written for each layout. A
// workgroup takes a 128 x 128 tile of x: sixteen lanes hold a row's 128 elements, eight
// each, so a row's maximum is a reduction over sixteen lanes; columns' maxima and the
// transposed bytes go through LDS. 16384 x 4096 bf16: along rows (no tiles) 30 us, 6.7 TB/s; along
// columns 33, 6.1 TB/s; both 46, 5.8 TB/s.
#include "pl_fp8.h"

namespace gadei::learner {
namespace {

constexpr int kBlock = 256;   // of quantize_rows
constexpr int kTile = 128;
// A thread takes four neighbouring rows of eight columns: with eight rows and half the threads, a
// few tiles take 7.4 us instead of 5.7 (57 x 900, both ways), many the same.
constexpr int kRows = 4, kThreads = kTile * kTile / 8 / kRows;

// Where word w (four rows) of column c of the transposed tile lies: fours of words exchanged by
// the column, so that neither the writes (16 columns eight apart, four words of each) nor
// the reads (four words of a column together) meet in a bank.
__device__ __forceinline__ int word_at(int c, int w) {
    return 32 * (c ^ ((c >> 6) & 1)) + (w ^ (((c >> 3) & 7) << 2));
}

// One matrix, or two of one type in a launch: the workgroups from blocks[0] on take the second's tiles.
struct Two {
    QuantArgs q[2];
    uint32_t tiles_x[2], blocks[2];
};

template <int X, bool SQUARE>
__global__ __launch_bounds__(kThreads) void quantize_tile(Two two) {
    const bool second = block_index() >= two.blocks[0];
    const QuantArgs &a = two.q[second];
    const uint32_t tiles_x = two.tiles_x[second], tile = block_index() - (second ? two.blocks[0] : 0);
    if (tile >= two.blocks[second]) return;
    using M = Mags<X>;
    constexpr int W = M::kWords;
    __shared__ uint32_t col_max[kTile];
    __shared__ __attribute__((aligned(16))) uint32_t columns[kTile * 32];
    __shared__ uint32_t all_max;
    const int64_t r0 = static_cast<int64_t>(tile / tiles_x) * kTile;
    const int64_t tile_x = tile % tiles_x, c0 = tile_x * kTile;
    const int g = threadIdx.x & 15, y = threadIdx.x >> 4;
    const int64_t col = c0 + 8 * g;
    const int count = a.cols - col >= 8 ? 8 : a.cols > col ? static_cast<int>(a.cols - col) : 0;
    const bool transposed = a.values_t != nullptr;
    if (threadIdx.x < kTile) col_max[threadIdx.x] = 0;
    if (threadIdx.x == 0) all_max = 0;

    auto row_of = [&](int i) { return r0 + kRows * y + i; };
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
        const uint32_t m = most_of_block(most8<X>(x[i]));
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
    for (int e = 0; e < 8; ++e) columns[word_at(8 * g + e, y)] = four_rows(x, e, as_scale(col_byte[e]));
    __syncthreads();
    const int64_t ld_t = (a.rows + 127) / 128 * 128;
    // 128 columns of x, 128 bytes each: eight lanes a column
#pragma unroll
    for (int i = threadIdx.x; i < kTile * 8; i += kThreads) {
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

// Along rows only: no tile is needed. A wave takes 512 columns of a row, four blocks and one word of
// scales, of kAlong rows.
constexpr int kAlong = 2;

template <int X>
__global__ __launch_bounds__(kBlock) void quantize_rows(QuantArgs a, uint32_t words) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t ld = (a.cols + 127) / 128 * 128;
    const uint32_t block = block_index(), word = block % words;
    const int64_t r0 = (static_cast<int64_t>(block / words) * (kBlock / 64) + wave) * kAlong;
    const int64_t col = 512ll * word + 8 * lane;
    if (col >= ld) return;   // whole blocks, whole sixteens of lanes
    const int count = a.cols - col >= 8 ? 8 : a.cols > col ? static_cast<int>(a.cols - col) : 0;
    Bits8<X> x[kAlong];
#pragma unroll
    for (int i = 0; i < kAlong; ++i) {
        const int64_t at = (r0 + i) * a.ld + col;
        if (r0 + i < a.rows && count == 8) x[i] = load8<X>(a.x, at);
        else x[i] = load8_some<X>(a.x, at, r0 + i < a.rows ? count : 0);
    }
#pragma unroll
    for (int i = 0; i < kAlong; ++i) {
        const uint32_t byte = scale_byte(most_of_block(most8<X>(x[i])));
        if (r0 + i >= a.rows) break;
        *reinterpret_cast<u32x2 *>(a.values + (r0 + i) * ld + col) =
            u32x2{four(x[i], 0, as_scale(byte)), four(x[i], 1, as_scale(byte))};
        if ((lane & 15) == 0)
            reinterpret_cast<uint8_t *>(a.scales + word * a.rows + r0 + i)[lane >> 4] =
                static_cast<uint8_t>(byte);
    }
}

}  // namespace

hipError_t launch_quantize(const QuantArgs &a, int dtype, bool square, hipStream_t s) {
    if (a.values_t == nullptr && !square) {
        const uint64_t words = (a.cols + 511) / 512;
        constexpr int kPer = kBlock / 64 * kAlong;   // rows of a workgroup
        const uint64_t blocks = words * ((a.rows + kPer - 1) / kPer);
        dim3 grid;
        if (!grid_of(blocks, kBlock, &grid)) return hipErrorInvalidConfiguration;
        const uint32_t w = static_cast<uint32_t>(words);
        if (dtype == PS_F32) quantize_rows<PS_F32><<<grid, kBlock, 0, s>>>(a, w);
        else quantize_rows<PS_BF16><<<grid, kBlock, 0, s>>>(a, w);
        return hipGetLastError();
    }
    return launch_quantize_two(a, QuantArgs{}, dtype, square, s);
}

hipError_t launch_quantize_two(const QuantArgs &a, const QuantArgs &b, int dtype, bool square,
                               hipStream_t s) {
    Two two{{a, b}, {}, {}};
    uint64_t all = 0;
    dim3 grid;
    for (int i = 0; i < 2; ++i) {
        const uint64_t x = (two.q[i].cols + kTile - 1) / kTile;
        const uint64_t blocks = x * ((two.q[i].rows + kTile - 1) / kTile);
        all += blocks;
        if (!grid_of(all, kThreads, &grid)) return hipErrorInvalidConfiguration;
        two.tiles_x[i] = static_cast<uint32_t>(x);
        two.blocks[i] = static_cast<uint32_t>(blocks);
    }
    if (all == 0) return hipSuccess;
    if (dtype == PS_F32) {
        if (square) quantize_tile<PS_F32, true><<<grid, kThreads, 0, s>>>(two);
        else quantize_tile<PS_F32, false><<<grid, kThreads, 0, s>>>(two);
    } else {
        if (square) quantize_tile<PS_BF16, true><<<grid, kThreads, 0, s>>>(two);
        else quantize_tile<PS_BF16, false><<<grid, kThreads, 0, s>>>(two);
    }
    return hipGetLastError();
}

}  // namespace gadei::learner
