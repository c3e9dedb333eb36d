// Streams over the rows of a matrix: embedding lookup and dropout.
//
// Mathematics: out[r, c] = keep(r, c) * factor * x[src(r), c], src(r) = r or ids[r].
// Bound by memory: every element is read once and written once. A thread takes eight
// consecutive columns (one evaluation of the generator, 20 wide products, gives their eight
// 16-bit numbers; the memory's time covers it) of one row or four, whose loads are issued
// together. Dropout of 16384 x 8192 bf16: 80 us, 6.7 TB/s of reads and writes; of 16384 x 4096
// fp32 79 us, 6.8 TB/s.
#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kBlock = 256;

// The block's threads cover 2^lx groups of eight columns times 256 / 2^lx rows.
template <int IDT, int X, int OUT, bool DROP, int ROWS, bool NT>
__global__ __launch_bounds__(kBlock) void rows_kernel(RowsArgs a, int lx, uint32_t tiles_x) {
    const uint32_t block = block_index(), tile_y = block / tiles_x, tile_x = block % tiles_x;
    const uint32_t group = (tile_x << lx) + (threadIdx.x & ((1u << lx) - 1));
    const uint32_t ny = kBlock >> lx;
    const uint64_t first = static_cast<uint64_t>(tile_y) * ny * ROWS + (threadIdx.x >> lx);
    const uint64_t col = 8ull * group;
    if (col >= a.cols) return;
    const int count = a.cols - col < 8 ? static_cast<int>(a.cols - col) : 8;
    // past the caches: 512 columns of one row, a wave's, at a time
    __shared__ f32x4 stage[NT && OUT == PS_F32 ? 2 * kBlock : 1];
    const bool lines = lx >= 6 && col - 8 * (threadIdx.x & 63) + 512 <= a.cols;

    int64_t src[ROWS];   // row of x; -1: zeros; -2: past the last row
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        const uint64_t r = first + u * ny;
        src[u] = -2;
        if (r < a.rows) {
            if constexpr (IDT == kNoIds) {
                src[u] = static_cast<int64_t>(r);
            } else {
                int64_t id;
                if constexpr (IDT == PL_I32) id = static_cast<const int32_t *>(a.ids)[r];
                else id = static_cast<const int64_t *>(a.ids)[r];
                src[u] = static_cast<uint64_t>(id) < a.vocab ? id : -1;
            }
        }
    }
    float x[ROWS][8];
    if (count == 8) {
        Bits8<X> bits[ROWS] = {};
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            if (src[u] >= 0) bits[u] = load8<X>(a.x, src[u] * a.x_ld + static_cast<int64_t>(col));
#pragma unroll
        for (int u = 0; u < ROWS; ++u) widen8<X>(x[u], bits[u]);
    } else {
#pragma unroll
        for (int u = 0; u < ROWS; ++u)
            load_some<X>(x[u], a.x, src[u] * a.x_ld + static_cast<int64_t>(col),
                         src[u] >= 0 ? count : 0);
    }
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        if (src[u] == -2) continue;
        const uint64_t r = first + u * ny;
        if constexpr (DROP) {
            drop8(x[u], a.factor, group, static_cast<uint32_t>(r), a.drop);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] *= a.factor;
        }
        if (src[u] == -1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = 0.0f;   // not factor * 0: the factor may be NaN
        }
        const int64_t at = static_cast<int64_t>(r) * a.out_ld + static_cast<int64_t>(col);
        if (NT && lines)
            store8_lines<OUT>(a.out, at, x[u], stage + (OUT == PS_F32 ? 2 * (threadIdx.x & ~63u) : 0));
        else if (count == 8) store8<OUT>(a.out, at, x[u]);
        else store_some<OUT>(a.out, at, x[u], count);
    }
}

template <int IDT, int X, int OUT, bool DROP, int ROWS, bool NT>
hipError_t launch_shape(const RowsArgs &a, int lx, hipStream_t s) {
    const uint64_t groups = (a.cols + 7) / 8;
    const uint64_t tiles_x = (groups + (1ull << lx) - 1) >> lx;
    const uint64_t rows = static_cast<uint64_t>(kBlock >> lx) * ROWS;
    const uint64_t blocks = tiles_x * ((a.rows + rows - 1) / rows);
    dim3 grid;
    if (!grid_of(blocks, kBlock, &grid)) return hipErrorInvalidConfiguration;
    rows_kernel<IDT, X, OUT, DROP, ROWS, NT><<<grid, kBlock, 0, s>>>(
        a, lx, static_cast<uint32_t>(tiles_x));
    return hipGetLastError();
}

// Four rows a thread keep enough loads under way for large matrices; small ones are over sooner with
// one, in more workgroups: 1824 lookups of 100 columns with dropout 3.6 us, 6.0 with four.
// Results that the caches (256 MB) will not hold for a reader go past them: 65536 lookups of 4096
// bf16 columns 129 us, 172 otherwise; dropout of 16384 x 8192 81 us, 93 otherwise.
template <int IDT, int X, int OUT, bool DROP>
hipError_t launch_drop(const RowsArgs &a, hipStream_t s) {
    const uint64_t groups = (a.cols + 7) / 8, all = groups * a.rows;
    int lx = 0;
    while (lx < 8 && (1ull << lx) < groups) ++lx;
    if (all <= 4ull * kCus * kBlock) return launch_shape<IDT, X, OUT, DROP, 1, false>(a, lx, s);
    if (8 * all * kBytes<OUT> <= kCached) return launch_shape<IDT, X, OUT, DROP, 4, false>(a, lx, s);
    return launch_shape<IDT, X, OUT, DROP, 4, true>(a, lx, s);
}

template <int IDT, int X, int OUT>
hipError_t launch(const RowsArgs &a, hipStream_t s) {
    return a.drop.drop != 0 ? launch_drop<IDT, X, OUT, true>(a, s) : launch_drop<IDT, X, OUT, false>(a, s);
}

template <int IDT>
hipError_t launch_typed(const RowsArgs &a, int x, int out, hipStream_t s) {
    if (x == PS_F32)
        return out == PS_F32 ? launch<IDT, PS_F32, PS_F32>(a, s) : launch<IDT, PS_F32, PS_BF16>(a, s);
    return out == PS_F32 ? launch<IDT, PS_BF16, PS_F32>(a, s) : launch<IDT, PS_BF16, PS_BF16>(a, s);
}

}  // namespace

hipError_t launch_rows(const RowsArgs &a, int id_type, int x, int out, hipStream_t s) {
    if (id_type == PL_I32) return launch_typed<PL_I32>(a, x, out, s);
    if (id_type == PL_I64) return launch_typed<PL_I64>(a, x, out, s);
    // dropout keeps its input's type
    return x == PS_F32 ? launch<kNoIds, PS_F32, PS_F32>(a, s)
                       : launch<kNoIds, PS_BF16, PS_BF16>(a, s);
}

}  // namespace gadei::learner
