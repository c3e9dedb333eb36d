// Gradient of an embedding table: out[v] = factor * sum of drop(grad[t]) over the
// tokens t with ids[t] == v.
//
// Summing by atomics would leave the order of a row's terms, and so its last bits,
// to chance, and would put a frequent token's thousands of terms in line for one address.
// Instead the tokens are sorted by id, stably, and every row is then summed in that order:
//
// sort    One workgroup per class of ids (id mod the number of classes) reads all
//         ids: it counts the ids of lower classes (where its part of the sorted list begins)
//         and its own per id, and on a second reading puts its tokens' positions
//         into their places. All workgroups read the same ids, which the L2s hold:
//         64k 4-byte ids are 256 KB per compute unit, and no pass over global memory
//         depends on another workgroup. Classes are residues, not ranges, because texts'
//         frequent ids are neighbours in many vocabularies.
// sum     A row of at most kPiece tokens is summed by the threads that write it (eight
//         columns each). The tokens of a longer row are cut into pieces of kPiece, whose
//         sums go to the workspace,
// join    and are added up in order by a last kernel.
//
// Bound by memory: grad is read once and out written once, rows without tokens included.
#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kSortThreads = 1024;
constexpr int kWaves = kSortThreads / 64;
constexpr int kMaxLocal = 1024;   // ids of one class
constexpr uint32_t kPiece = 64;   // tokens that one thread adds up

struct Row {
    uint32_t begin, count;   // its part of the sorted list
};
struct Piece {
    uint32_t row, begin, count;   // count 0: none
    uint32_t of;                  // the first piece of a row: how many it has; others 0
};

struct Plan {
    int class_bits;
    uint32_t classes, local;   // ids of a class, rounded up
    uint32_t pieces;           // room for
    size_t rows_at, perm_at, pieces_at, sums_at, bytes;
};

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

Plan make_plan(int64_t tokens, int64_t vocab, int64_t dim) {
    Plan p{};
    // at least one class per compute unit, and no more ids in a class than the
    // counters in LDS
    p.class_bits = 8;
    while (((vocab - 1) >> p.class_bits) >= kMaxLocal) ++p.class_bits;
    p.classes = 1u << p.class_bits;
    p.local = static_cast<uint32_t>((vocab + p.classes - 1) >> p.class_bits);
    // a row with c > kPiece tokens has ceil(c / kPiece) < 2 c / kPiece pieces
    p.pieces = static_cast<uint32_t>(2 * tokens / kPiece);
    p.rows_at = 0;
    p.perm_at = align256(sizeof(Row) * p.classes * size_t(p.local));
    p.pieces_at = p.perm_at + align256(sizeof(uint32_t) * size_t(tokens));
    p.sums_at = p.pieces_at + align256(sizeof(Piece) * size_t(p.pieces));
    p.bytes = p.sums_at + sizeof(float) * size_t(p.pieces) * size_t(dim);
    return p;
}

template <int IDT>
__device__ __forceinline__ uint32_t load_id(const void *ids, uint32_t t, uint32_t vocab) {
    // ids that are no token become 2^32 - 1 (vocab is at most 2^31)
    if constexpr (IDT == PL_I32) {
        const uint32_t id = static_cast<const uint32_t *>(ids)[t];
        return id < vocab ? id : 0xffffffffu;
    } else {
        const uint64_t id = static_cast<const uint64_t *>(ids)[t];
        return id < vocab ? static_cast<uint32_t>(id) : 0xffffffffu;
    }
}

// Sum of x over the workgroup's lanes before this one; `total` is all of them.
__device__ __forceinline__ uint32_t scan_exclusive(uint32_t x, uint32_t *wave_sums, uint32_t &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t sum = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(sum, d);
        if (lane >= d) sum += y;
    }
    if (lane == 63) wave_sums[wave] = sum;
    __syncthreads();
    uint32_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t y = wave_sums[w];
        if (w < wave) before += y;
        all += y;
    }
    __syncthreads();
    total = all;
    return before + sum - x;
}

constexpr int kAhead = 8;   // ids that a thread loads together

template <int IDT>
__global__ __launch_bounds__(kSortThreads) void sort_tokens(const void *ids, uint32_t tokens,
                                                            uint32_t vocab, int class_bits,
                                                            uint32_t local, Row *rows, uint32_t *perm,
                                                            Piece *pieces) {
    __shared__ uint32_t counts[kWaves][kMaxLocal];   // of each wave's part of the ids
    __shared__ uint32_t wave_sums[kWaves];
    const uint32_t mine = blockIdx.x, mask = (1u << class_bits) - 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (uint32_t i = threadIdx.x; i < kWaves * kMaxLocal; i += kSortThreads) (&counts[0][0])[i] = 0;
    __syncthreads();

    // a wave's part of the ids: a run of whole steps of 64
    const uint32_t steps = (tokens + 64 * kWaves - 1) / (64 * kWaves);
    const uint64_t part = static_cast<uint64_t>(wave) * steps * 64;
    uint32_t lower = 0;
    for (uint32_t s = 0; s < steps; s += kAhead) {
        uint32_t id[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint64_t t = part + (s + j) * 64ull + lane;
            id[j] = s + j < steps && t < tokens
                        ? load_id<IDT>(ids, static_cast<uint32_t>(t), vocab) : 0xffffffffu;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (id[j] == 0xffffffffu) continue;
            const uint32_t c = id[j] & mask;
            lower += c < mine;
            if (c == mine) atomicAdd(&counts[wave][id[j] >> class_bits], 1u);
        }
    }
    __syncthreads();

    uint32_t base, total;
    (void)scan_exclusive(lower, wave_sums, base);   // every class below comes before
    // thread l: the class's id l. Its tokens by wave, then where each wave's begin
    const uint32_t l = threadIdx.x;
    uint32_t count = 0;
    if (l < local)
        for (int w = 0; w < kWaves; ++w) count += counts[w][l];
    const uint32_t begin = base + scan_exclusive(count, wave_sums, total);
    if (l < local) {
        uint32_t at = begin;
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = counts[w][l];
            counts[w][l] = at;
            at += c;
        }
        rows[static_cast<uint64_t>(mine) * local + l] = Row{begin, count};
    }
    // the pieces of long rows, in the class's part of the list of pieces
    const uint32_t n = count > kPiece ? (count + kPiece - 1) / kPiece : 0;
    const uint32_t from = static_cast<uint32_t>(2ull * base / kPiece);
    // the last one goes on to the list's end: ids that are no token are in no class
    const uint32_t to = static_cast<uint32_t>(
        2ull * (mine == mask ? tokens : base + total) / kPiece);
    uint32_t used;
    const uint32_t slot = from + scan_exclusive(n, wave_sums, used);   // and orders counts[]
    for (uint32_t i = 0; i < n; ++i) {
        const uint32_t done = i * kPiece;
        pieces[slot + i] = Piece{(l << class_bits) | mine, begin + done,
                                 count - done < kPiece ? count - done : kPiece, i == 0 ? n : 0};
    }
    for (uint32_t i = from + used + threadIdx.x; i < to; i += kSortThreads)
        pieces[i] = Piece{0, 0, 0, 0};

    // second reading: positions into their places, in order within a wave's part
    if (total == 0) return;
    for (uint32_t s = 0; s < steps; s += kAhead) {
        uint32_t id[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const uint64_t t = part + (s + j) * 64ull + lane;
            id[j] = s + j < steps && t < tokens
                        ? load_id<IDT>(ids, static_cast<uint32_t>(t), vocab) : 0xffffffffu;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            uint64_t todo = __ballot(id[j] != 0xffffffffu && (id[j] & mask) == mine);
            while (todo) {   // one id after the other: all its lanes at once
                const uint32_t one = __shfl(id[j], __ffsll(static_cast<unsigned long long>(todo)) - 1);
                const bool same = id[j] == one;
                const uint64_t lanes = __ballot(same);
                const uint32_t at = counts[wave][one >> class_bits];
                if (same)
                    perm[at + __popcll(lanes & ((1ull << lane) - 1))] =
                        static_cast<uint32_t>(part + (s + j) * 64ull + lane);
                counts[wave][one >> class_bits] = at + __popcll(lanes);   // all lanes alike
                todo &= ~lanes;
            }
        }
    }
}

constexpr int kBlock = 256;

// sum += drop(grad[t]) over `count` tokens of the sorted list, columns col .. col+7.
template <int G, bool DROP>
__device__ __forceinline__ void add_tokens(float (&sum)[8], const GradArgs &a, const uint32_t *perm,
                                           uint32_t count, uint32_t group, int columns) {
    constexpr uint32_t kTogether = 4;
    const int64_t col = 8ll * group;
    for (uint32_t i = 0; i < count; i += kTogether) {
        uint32_t t[kTogether];
        float x[kTogether][8];
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j) t[j] = perm[i + j < count ? i + j : i];
        if (columns == 8) {
            Bits8<G> bits[kTogether];
#pragma unroll
            for (uint32_t j = 0; j < kTogether; ++j) bits[j] = load8<G>(a.grad, t[j] * a.grad_ld + col);
#pragma unroll
            for (uint32_t j = 0; j < kTogether; ++j) widen8<G>(x[j], bits[j]);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kTogether; ++j)
                load_some<G>(x[j], a.grad, t[j] * a.grad_ld + col, columns);
        }
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j) {
            if (i + j >= count) break;
            if constexpr (DROP) drop8(x[j], 1.0f, group, t[j], a.drop);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[j][e];
        }
    }
}

template <int OUT>
__device__ __forceinline__ void write_row(const GradArgs &a, float (&sum)[8], uint32_t row,
                                          uint32_t group, int columns) {
    const int64_t at = row * a.out_ld + 8ll * group;
    float old[8];
    if (a.accumulate) {
        if (columns == 8) widen8<OUT>(old, load8<OUT>(a.out, at));
        else load_some<OUT>(old, a.out, at, columns);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sum[e] *= a.factor;
        if (a.accumulate) sum[e] += old[e];
    }
    if (columns == 8) store8<OUT>(a.out, at, sum);
    else store_some<OUT>(a.out, at, sum, columns);
}

// Blocks of 2^lx groups of eight columns times 256 / 2^lx rows or pieces: first the pieces,
// which take longest, then the rows.
template <int G, int OUT, bool DROP>
__global__ __launch_bounds__(kBlock) void sum_rows(GradArgs a, Plan p, int lx, uint32_t tiles_x,
                                                   uint32_t piece_blocks) {
    const char *ws = static_cast<const char *>(a.workspace);
    const uint32_t *perm = reinterpret_cast<const uint32_t *>(ws + p.perm_at);
    const uint32_t ny = kBlock >> lx;
    const bool pieces = blockIdx.x < piece_blocks;
    const uint32_t block = pieces ? blockIdx.x : blockIdx.x - piece_blocks;
    const uint32_t group = ((block % tiles_x) << lx) + (threadIdx.x & ((1u << lx) - 1));
    const uint64_t y = static_cast<uint64_t>(block / tiles_x) * ny + (threadIdx.x >> lx);
    const uint64_t col = 8ull * group;
    if (col >= a.dim) return;
    const int columns = a.dim - col < 8 ? static_cast<int>(a.dim - col) : 8;
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (pieces) {
        if (y >= p.pieces) return;
        const Piece piece = reinterpret_cast<const Piece *>(ws + p.pieces_at)[y];
        if (piece.count == 0) return;
        add_tokens<G, DROP>(sum, a, perm + piece.begin, piece.count, group, columns);
        float *sums = reinterpret_cast<float *>(static_cast<char *>(a.workspace) + p.sums_at);
        const int64_t at = static_cast<int64_t>(y * a.dim + col);
        if (columns == 8) store8<PS_F32>(sums, at, sum);
        else store_some<PS_F32>(sums, at, sum, columns);
        return;
    }
    if (y >= a.vocab) return;
    const uint32_t v = static_cast<uint32_t>(y);
    const Row row = reinterpret_cast<const Row *>(ws + p.rows_at)[
        static_cast<uint64_t>(v & (p.classes - 1)) * p.local + (v >> p.class_bits)];
    if (row.count > kPiece || (row.count == 0 && a.accumulate)) return;
    add_tokens<G, DROP>(sum, a, perm + row.begin, row.count, group, columns);
    write_row<OUT>(a, sum, v, group, columns);
}

// The rows cut into pieces: their sums, in order.
template <int OUT>
__global__ __launch_bounds__(kBlock) void join_pieces(GradArgs a, Plan p, int lx, uint32_t tiles_x) {
    const char *ws = static_cast<const char *>(a.workspace);
    const uint32_t group = ((blockIdx.x % tiles_x) << lx) + (threadIdx.x & ((1u << lx) - 1));
    const uint64_t y = static_cast<uint64_t>(blockIdx.x / tiles_x) * (kBlock >> lx) + (threadIdx.x >> lx);
    const uint64_t col = 8ull * group;
    if (col >= a.dim || y >= p.pieces) return;
    const Piece piece = reinterpret_cast<const Piece *>(ws + p.pieces_at)[y];
    if (piece.of == 0) return;
    const int columns = a.dim - col < 8 ? static_cast<int>(a.dim - col) : 8;
    const float *sums = reinterpret_cast<const float *>(ws + p.sums_at);
    float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (uint32_t i = 0; i < piece.of; ++i) {
        float x[8];
        const int64_t at = static_cast<int64_t>((y + i) * a.dim + col);
        if (columns == 8) widen8<PS_F32>(x, load8<PS_F32>(sums, at));
        else load_some<PS_F32>(x, sums, at, columns);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[e] += x[e];
    }
    write_row<OUT>(a, sum, piece.row, group, columns);
}

template <int G, int OUT>
hipError_t launch_sums(const GradArgs &a, const Plan &p, hipStream_t s) {
    const uint64_t groups = (a.dim + 7) / 8;
    int lx = 0;
    while (lx < 8 && (1ull << lx) < groups) ++lx;
    const uint32_t tiles_x = static_cast<uint32_t>((groups + (1ull << lx) - 1) >> lx);
    const uint32_t ny = kBlock >> lx;
    const uint64_t piece_blocks = static_cast<uint64_t>((p.pieces + ny - 1) / ny) * tiles_x;
    const uint64_t blocks = piece_blocks + (static_cast<uint64_t>(a.vocab) + ny - 1) / ny * tiles_x;
    if (blocks > 0xffffffffull / kBlock) return hipErrorInvalidConfiguration;
    const uint32_t pb = static_cast<uint32_t>(piece_blocks);
    if (a.drop.drop != 0)
        sum_rows<G, OUT, true><<<static_cast<uint32_t>(blocks), kBlock, 0, s>>>(a, p, lx, tiles_x, pb);
    else
        sum_rows<G, OUT, false><<<static_cast<uint32_t>(blocks), kBlock, 0, s>>>(a, p, lx, tiles_x, pb);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || pb == 0) return e;
    join_pieces<OUT><<<pb, kBlock, 0, s>>>(a, p, lx, tiles_x);
    return hipGetLastError();
}

}  // namespace

size_t grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    return make_plan(tokens, vocab, dim).bytes;
}

hipError_t launch_grad(const GradArgs &a, int id_type, int grad_dtype, int out_dtype,
                       hipStream_t s) {
    const Plan p = make_plan(a.tokens, a.vocab, static_cast<int64_t>(a.dim));
    char *ws = static_cast<char *>(a.workspace);
    Row *rows = reinterpret_cast<Row *>(ws + p.rows_at);
    uint32_t *perm = reinterpret_cast<uint32_t *>(ws + p.perm_at);
    Piece *pieces = reinterpret_cast<Piece *>(ws + p.pieces_at);
    if (id_type == PL_I32)
        sort_tokens<PL_I32><<<p.classes, kSortThreads, 0, s>>>(a.ids, a.tokens, a.vocab, p.class_bits,
                                                               p.local, rows, perm, pieces);
    else
        sort_tokens<PL_I64><<<p.classes, kSortThreads, 0, s>>>(a.ids, a.tokens, a.vocab, p.class_bits,
                                                               p.local, rows, perm, pieces);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (grad_dtype == PS_F32)
        return out_dtype == PS_F32 ? launch_sums<PS_F32, PS_F32>(a, p, s)
                                   : launch_sums<PS_F32, PS_BF16>(a, p, s);
    return out_dtype == PS_F32 ? launch_sums<PS_BF16, PS_F32>(a, p, s)
                               : launch_sums<PS_BF16, PS_BF16>(a, p, s);
}

}  // namespace gadei::learner
