// Gradient of an embedding table: out[v] = factor * sum of drop(grad[t]) over the
// tokens t with ids[t] == v.
//
// Summing by atomics would leave the order of a row's terms, and so its last bits,
// to chance, and would put a frequent token's thousands of terms in line for one address.
// Instead the tokens are sorted by id, stably, and every row is then summed in that order:
//
// sort    One workgroup per class of ids (id mod the number of classes) reads all
//         ids: it counts the ids of lower classes (where its part of the sorted list begins)
//         and its own per id, writes its tokens down, and then puts their positions
//         into their places. All workgroups read the same ids, which the L2s hold:
//         64k 4-byte ids are 256 KB per compute unit, and no pass over global memory
//         depends on another workgroup. Classes are residues, not ranges, because texts'
//         frequent ids are neighbours in many vocabularies.
// sum     A row of at most `piece` tokens is summed by the threads that write it (eight
//         columns each). The tokens of a longer row are cut into pieces of that many, whose
//         sums go to the workspace,
// join    and are added up in order by a last kernel.
//
// Where there are few tokens, launches and latencies take longest, and one kernel does all of it
// (sum_few).
//
// Bound by memory: grad is read once and out written once, rows without tokens included. 65536
// tokens of 4096 bf16 columns into 65536 fp32 rows, with dropout (1.6 GB): 360 us, of which sort 27,
// sum 330 (4.9 TB/s) and join 13; 1824 tokens of 100 fp32 columns into 50000 rows in one launch of 15.
#include <algorithm>

#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kMaxLocal = 1024;   // ids of one class
constexpr uint32_t kMaxFound = 1024;   // tokens that a wave writes down
// Of long lists of ids nothing is written down, as a frequent id's tokens are too many: the call over
// 65536 ids of 50000, of 16 columns, takes 44 us with writing and 50 without, over 200000 89 and 98, but
// over 262144 160 and 119.
constexpr uint32_t kNoted = 1 << 17;
constexpr int kPlaceBits = 22;   // of a token in a wave's part of the ids; the rest hold the id in its class
static_assert(kMaxLocal <= 1 << (32 - kPlaceBits) && kNoted <= 1 << kPlaceBits, "a word each");

struct Row {
    uint32_t begin, count;   // its part of the sorted list
};
struct Piece {
    uint32_t row, begin, count;   // count 0: none
    uint32_t of;                  // the first piece of a row: how many it has; others 0
};

struct Plan {
    int class_bits;
    uint32_t piece;            // tokens that one thread adds up
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
    // One token after another is latency, and pieces are traffic of their own. In us, with dropout,
    // with pieces of 8 and of 32: 65536 tokens of 100 columns 60 and 69, 32768 of 1000 95 and 93,
    // 65536 of 1200 169 and 157, 65536 of 4096 406 and 364 (of 64 367).
    p.piece = tokens * dim < (int64_t(1) << 25) ? 8 : 32;
    // a row with c > piece tokens has ceil(c / piece) < 2 c / piece pieces
    p.pieces = tokens <= p.piece ? 0 : static_cast<uint32_t>(2 * tokens / p.piece);
    p.rows_at = 0;
    p.perm_at = align256(sizeof(Row) * p.classes * size_t(p.local));
    p.pieces_at = p.perm_at + align256(sizeof(uint32_t) * size_t(tokens));
    p.sums_at = p.pieces_at + align256(sizeof(Piece) * size_t(p.pieces));
    p.bytes = p.sums_at + sizeof(float) * size_t(p.pieces) * size_t(dim);
    return p;
}

// Ids as unsigned numbers: negative ones are no tokens like all that are too large (vocab is
// at most 2^31).
template <int IDT> struct IdBits { using type = uint32_t; };
template <> struct IdBits<PL_I64> { using type = uint64_t; };

// Sum of x over the lanes of the workgroup's WAVES waves before this one; `total` is all of them.
template <int WAVES>
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
    for (int w = 0; w < WAVES; ++w) {
        const uint32_t y = wave_sums[w];
        if (w < wave) before += y;
        all += y;
    }
    __syncthreads();
    total = all;
    return before + sum - x;
}

constexpr int kAhead = 8;   // steps whose ids are loaded together

// Calls f(step, id) for a wave's steps first, first + 1, .. of 64 ids, in order; ids past the last
// are 2^32 - 1.
template <int IDT, class F>
__device__ __forceinline__ void each_id(const void *ids, uint32_t tokens, uint32_t first, uint32_t steps,
                                        int lane, F f) {
    for (uint32_t s = 0; s < steps; s += kAhead) {
        const uint64_t t0 = 64ull * (first + s);
        typename IdBits<IDT>::type raw[kAhead];
        const auto *p = static_cast<const typename IdBits<IDT>::type *>(ids) + t0 + lane;
        if (s + kAhead <= steps && t0 + 64 * kAhead <= tokens) {   // the same for the whole wave
#pragma unroll
            for (int j = 0; j < kAhead; ++j) raw[j] = p[64 * j];
        } else {
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                raw[j] = ~typename IdBits<IDT>::type(0);
                if (s + j < steps && t0 + 64 * j + lane < tokens) raw[j] = p[64 * j];
            }
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) f(first + s + j, raw[j]);
    }
}

// Puts the positions of some of a wave's lanes (those with a bit in `todo`, one at least) where the
// next ones of their ids belong; next[local] is where, and moves on. The lanes of an id, its rank
// among them and how many they are come from ballots, one id after the other; LDS is asked for all
// ids at once.
__device__ __forceinline__ void put(uint32_t *next, uint32_t *list, uint64_t todo, uint32_t local,
                                    uint32_t position, int lane) {
    const bool mine = todo >> lane & 1;
    uint32_t rank = 0, many = 0;
    int first = lane;
    while (todo) {
        const int f = __ffsll(static_cast<unsigned long long>(todo)) - 1;
        const uint32_t one = __builtin_amdgcn_readlane(local, f);
        const uint64_t lanes = todo & __ballot(local == one);
        if (lanes >> lane & 1) {
            rank = __popcll(lanes & ((1ull << lane) - 1));
            many = __popcll(lanes);
            first = f;
        }
        todo &= ~lanes;
    }
    uint32_t at = 0;
    if (mine && first == lane) at = atomicAdd(&next[local], many);
    at = __shfl(at, first);
    if (mine) list[at + rank] = position;
}

// A row that is cut into pieces, which lie in the list of pieces from `slot` on.
struct LongRow {
    uint32_t row, begin, count, slot;
};
constexpr uint32_t kLongRows = 64;   // of a class, whose pieces all threads write

__device__ __forceinline__ void write_pieces(const LongRow &r, uint32_t piece, Piece *pieces, uint32_t i,
                                             uint32_t step) {
    const uint32_t n = (r.count + piece - 1) / piece;
    for (; i < n; i += step)
        pieces[r.slot + i] =
            Piece{r.row, r.begin + i * piece, min(piece, r.count - i * piece), i == 0 ? n : 0};
}

// WAVES waves; a thread does the bookkeeping of kMaxLocal / (64 WAVES) ids.
template <int IDT, int WAVES, bool NOTED>
__global__ __launch_bounds__(64 * WAVES) void sort_tokens(const void *ids, uint32_t tokens, uint32_t vocab,
                                                          Plan p, Row *rows, uint32_t *perm,
                                                          Piece *pieces) {
    using Id = typename IdBits<IDT>::type;
    constexpr int kEach = kMaxLocal / (64 * WAVES);
    __shared__ uint32_t counts[WAVES][kMaxLocal];   // of each wave's part of the ids
    // tokens of the class, in order: id in the class, place in the part
    __shared__ uint32_t found[WAVES][NOTED ? kMaxFound : 1];
    __shared__ uint32_t wave_sums[WAVES];
    __shared__ LongRow longs[kLongRows];
    __shared__ uint32_t n_longs;
    const uint32_t mine = blockIdx.x, mask = p.classes - 1;
    const int class_bits = p.class_bits;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (uint32_t l = threadIdx.x; l < p.local; l += 64 * WAVES)
        for (int w = 0; w < WAVES; ++w) counts[w][l] = 0;
    if (threadIdx.x == 0) n_longs = 0;
    __syncthreads();

    // A wave's part of the ids is a run of whole steps of 64. Few instructions an id: what this
    // kernel takes is the ids times them, on every compute unit.
    const uint32_t steps = (tokens + 64 * WAVES - 1) / (64 * WAVES), first = wave * steps;
    uint32_t lower = 0, n_found = 0;
    each_id<IDT>(ids, tokens, first, steps, lane, [&](uint32_t step, Id id) {
        const bool real = id < vocab;
        const uint32_t low = static_cast<uint32_t>(id), c = low & mask;
        lower += __popcll(__ballot(real && c < mine));   // in scalar registers
        const bool hit = real && c == mine;
        const uint64_t hits = NOTED ? __ballot(hit) : 1;
        if (hits == 0) return;
        // many of one id are one addition: LDS would take them one after another
        const int leader = __ffsll(static_cast<unsigned long long>(hits)) - 1;
        const uint32_t leads = __builtin_amdgcn_readlane(low, leader);
        const uint64_t alike = NOTED ? hits & __ballot(low == leads) : 0;
        if (hit) {
            const uint32_t n = alike >> lane & 1 ? static_cast<uint32_t>(__popcll(alike)) : 1u;
            if (n == 1 || lane == leader) atomicAdd(&counts[wave][low >> class_bits], n);
            const uint32_t i = n_found + __popcll(hits & ((1ull << lane) - 1));
            if (NOTED && i < kMaxFound)
                found[wave][i] = (low >> class_bits) << kPlaceBits | ((step - first) * 64 + lane);
        }
        n_found += __popcll(hits);
    });
    __syncthreads();

    uint32_t base, total;
    (void)scan_exclusive<WAVES>(lane == 0 ? lower : 0, wave_sums, base);   // every class below comes before
    // tokens of a thread's ids, then where each wave's tokens of each id begin
    const uint32_t l0 = threadIdx.x * kEach;
    uint32_t count[kEach], all = 0, n[kEach], all_pieces = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        count[e] = 0;
        if (l0 + e < p.local)
            for (int w = 0; w < WAVES; ++w) count[e] += counts[w][l0 + e];
        all += count[e];
        n[e] = count[e] > p.piece ? (count[e] + p.piece - 1) / p.piece : 0;
        all_pieces += n[e];
    }
    uint32_t at = base + scan_exclusive<WAVES>(all, wave_sums, total);
    // the pieces of long rows lie in the class's part of the list of pieces; the last class's
    // goes on to the list's end: ids that are no token are in no class
    uint32_t used = 0, slot = 0, from = 0;
    if (p.pieces != 0) {
        from = static_cast<uint32_t>(2ull * base / p.piece);
        slot = from + scan_exclusive<WAVES>(all_pieces, wave_sums, used);
    }
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const uint32_t l = l0 + e;
        if (l >= p.local) break;
        rows[static_cast<uint64_t>(mine) * p.local + l] = Row{at, count[e]};
        if (n[e] != 0) {
            const LongRow row = {(l << class_bits) | mine, at, count[e], slot};
            const uint32_t i = n[e] > 4 ? atomicAdd(&n_longs, 1u) : kLongRows;
            if (i < kLongRows) longs[i] = row;
            else write_pieces(row, p.piece, pieces, 0, 1);
        }
        slot += n[e];
        for (int w = 0; w < WAVES; ++w) {
            const uint32_t c = counts[w][l];
            counts[w][l] = at;
            at += c;
        }
    }
    __syncthreads();
    for (uint32_t i = 0; i < min(n_longs, kLongRows); ++i)
        write_pieces(longs[i], p.piece, pieces, threadIdx.x, 64 * WAVES);
    if (p.pieces != 0) {
        const uint32_t to = mine == mask ? p.pieces : static_cast<uint32_t>(2ull * (base + total) / p.piece);
        for (uint32_t i = from + used + threadIdx.x; i < to; i += 64 * WAVES) pieces[i] = Piece{0, 0, 0, 0};
    }

    // Positions into their places, in order within a wave's part: those that were written down, or,
    // where they were too many (in a frequent id's class), found again.
    if (total == 0) return;
    if (NOTED && n_found <= kMaxFound) {
        for (uint32_t i = 0; i < n_found; i += 64) {
            const uint32_t token = i + lane < n_found ? found[wave][i + lane] : 0;
            put(counts[wave], perm, __ballot(i + lane < n_found), token >> kPlaceBits,
                first * 64 + (token & ((1u << kPlaceBits) - 1)), lane);
        }
        return;
    }
    each_id<IDT>(ids, tokens, first, steps, lane, [&](uint32_t step, Id id) {
        const uint32_t low = static_cast<uint32_t>(id);
        uint64_t todo = __ballot(id < vocab && (low & mask) == mine);
        while (todo) {   // one id after the other: all its lanes at once
            const int f = __ffsll(static_cast<unsigned long long>(todo)) - 1;
            const uint32_t one = __builtin_amdgcn_readlane(low, f);
            const uint64_t lanes = todo & __ballot(low == one);
            const uint32_t at = counts[wave][one >> class_bits];
            if (lanes >> lane & 1)
                perm[at + __popcll(lanes & ((1ull << lane) - 1))] = step * 64 + lane;
            counts[wave][one >> class_bits] = at + __popcll(lanes);   // all lanes alike
            todo &= ~lanes;
        }
    });
}

constexpr int kBlock = 256;

// sum += drop(grad[t]) over `count` tokens of the sorted list, columns col .. col+7.
template <int G, bool DROP>
__device__ __forceinline__ void add_tokens(float (&sum)[8], const GradArgs &a, const uint32_t *perm,
                                           uint32_t count, uint32_t group, int columns) {
    // four tokens' loads together: eight leave room for fewer waves (407 us instead of 363 for 65536
    // tokens of 4096 columns)
    constexpr uint32_t kTogether = 4;
    const int64_t col = 8ll * group;
    for (uint32_t i = 0; i < count; i += kTogether) {
        uint32_t t[kTogether];
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j) t[j] = perm[i + j < count ? i + j : i];
        Bits8<G> bits[kTogether] = {};
        if (columns == 8) {
#pragma unroll
            for (uint32_t j = 0; j < kTogether; ++j)
                if (i + j < count) bits[j] = load8<G>(a.grad, t[j] * a.grad_ld + col);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < kTogether; ++j)
                if (i + j < count) bits[j] = load8_some<G>(a.grad, t[j] * a.grad_ld + col, columns);
        }
#pragma unroll
        for (uint32_t j = 0; j < kTogether; ++j) {
            if (i + j >= count) break;
            float x[8];
            widen8<G>(x, bits[j]);
            if constexpr (DROP) drop8(x, 1.0f, group, t[j], a.drop);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += x[e];
        }
    }
}

// A result past the caches (true: of a table too large for them) whose 512 columns from the wave's
// first on are one row's and inside it: stage is the wave's part of LDS. Otherwise null.
// A row without tokens (the sums are zeros) is zeros even where the factor is not finite.
template <int OUT>
__device__ __forceinline__ void write_row(const GradArgs &a, float (&sum)[8], uint32_t tokens, uint32_t row,
                                          uint32_t group, int columns, f32x4 *stage = nullptr) {
    const float factor = tokens != 0 ? a.factor : 0.0f;
    const int64_t at = row * a.out_ld + 8ll * group;
    float old[8];
    if (a.accumulate) {
        if (columns == 8) widen8<OUT>(old, load8<OUT>(a.out, at));
        else load_some<OUT>(old, a.out, at, columns);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        sum[e] *= factor;
        if (a.accumulate) sum[e] += old[e];
    }
    if (stage != nullptr) store8_lines<OUT>(a.out, at, sum, stage);
    else if (columns == 8) store8<OUT>(a.out, at, sum);
    else store_some<OUT>(a.out, at, sum, columns);
}

// Blocks of 2^lx groups of eight columns times 256 / 2^lx pieces or rows: first the pieces, which
// take longest, then the rows.
template <int G, int OUT, bool DROP>
__global__ __launch_bounds__(kBlock) void sum_rows(GradArgs a, Plan p, int lx, uint32_t tiles_x,
                                                   uint32_t piece_blocks, bool past_caches) {
    __shared__ f32x4 stage[OUT == PS_F32 ? 2 * kBlock : 1];
    const char *ws = static_cast<const char *>(a.workspace);
    const uint32_t *perm = reinterpret_cast<const uint32_t *>(ws + p.perm_at);
    const bool pieces = block_index() < piece_blocks;
    const uint32_t block = pieces ? block_index() : block_index() - piece_blocks;
    const uint32_t group = ((block % tiles_x) << lx) + (threadIdx.x & ((1u << lx) - 1));
    const uint64_t y = static_cast<uint64_t>(block / tiles_x) * (kBlock >> lx) + (threadIdx.x >> lx);
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
    if (row.count > p.piece || (row.count == 0 && a.accumulate)) return;
    add_tokens<G, DROP>(sum, a, perm + row.begin, row.count, group, columns);
    // lx >= 6: a wave's lanes are of one row
    const bool lines = past_caches && lx >= 6 && col - 8 * (threadIdx.x & 63) + 512 <= a.dim;
    write_row<OUT>(a, sum, row.count, v, group, columns,
                   lines ? stage + (OUT == PS_F32 ? 2 * (threadIdx.x & ~63u) : 0) : nullptr);
}

// The rows cut into pieces: their sums, in a fixed order. A workgroup takes kJoinSlots pieces of the list
// after one another, most of which begin no row; where one does, the threads of one column share
// its pieces, a run each, and the runs' sums are added up in halves.
constexpr int kJoinMostGroups = 4;   // log2 of the groups of columns of a workgroup, at most
constexpr uint32_t kJoinSlots = 16;

template <int OUT>
__global__ __launch_bounds__(kBlock) void join_pieces(GradArgs a, Plan p, int lx, uint32_t tiles_x) {
    __shared__ float runs[kBlock][8];
    const char *ws = static_cast<const char *>(a.workspace);
    const Piece *list = reinterpret_cast<const Piece *>(ws + p.pieces_at);
    const float *sums = reinterpret_cast<const float *>(ws + p.sums_at);
    const uint32_t run = threadIdx.x >> lx, n_runs = kBlock >> lx;
    const uint32_t group = (blockIdx.x % tiles_x << lx) + (threadIdx.x & ((1u << lx) - 1));
    const uint64_t col = 8ull * group;
    const int columns = col >= a.dim ? 0 : a.dim - col < 8 ? static_cast<int>(a.dim - col) : 8;
    const uint32_t slot = blockIdx.x / tiles_x * kJoinSlots, lane = threadIdx.x & 63;
    const uint32_t mine = lane < kJoinSlots && slot + lane < p.pieces ? list[slot + lane].of : 0;
    for (uint64_t todo = __ballot(mine != 0); todo != 0; todo &= todo - 1) {   // the same for all waves
        const int first = __ffsll(static_cast<unsigned long long>(todo)) - 1;
        const uint32_t y = slot + first, of = __builtin_amdgcn_readlane(mine, first);
        const uint32_t each = (of + n_runs - 1) / n_runs;
        const uint32_t from = min(run * each, of), to = min(from + each, of);
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (columns != 0) {
#pragma unroll 4
            for (uint32_t i = from; i < to; ++i) {
                float x[8];
                const int64_t at = static_cast<int64_t>((y + i) * a.dim + col);
                if (columns == 8) widen8<PS_F32>(x, load8<PS_F32>(sums, at));
                else load_some<PS_F32>(x, sums, at, columns);
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += x[e];
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) runs[threadIdx.x][e] = sum[e];
        __syncthreads();
        for (uint32_t half = n_runs / 2; half != 0; half /= 2) {
            if (run < half) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[e] += runs[threadIdx.x + (half << lx)][e];
                    runs[threadIdx.x][e] = sum[e];
                }
            }
            __syncthreads();
        }
        if (run == 0 && columns != 0) write_row<OUT>(a, sum, of, list[y].row, group, columns);
    }
}

// Few tokens and narrow rows: everything in one launch. A workgroup takes kSmallRows rows of the
// table and up to 128 columns; it reads all ids and lists its rows' tokens in LDS, in order, as
// sort_tokens does. A row of more than kSmallAlone tokens is shared by all threads of a column, a
// run of its tokens each, and their sums are added up in order.
constexpr uint32_t kSmallTokens = 4096, kSmallRows = 64, kSmallAlone = 4;
constexpr int kSmallWaves = kBlock / 64;

template <int IDT, int G, int OUT, bool DROP>
__global__ __launch_bounds__(kBlock) void sum_few(GradArgs a, int lx, uint32_t tiles_x) {
    using Id = typename IdBits<IDT>::type;
    constexpr int kSteps = kSmallTokens / kBlock;   // ids of a lane
    __shared__ uint32_t counts[kSmallWaves][kSmallRows], begins[kSmallRows + 1], list[kSmallTokens];
    __shared__ float runs[kBlock][8];
    __shared__ uint64_t shared_rows;   // bit r: row r is
    const uint32_t v0 = block_index() / tiles_x * kSmallRows;
    if (v0 >= a.vocab) return;
    const uint32_t x = threadIdx.x & ((1u << lx) - 1), y = threadIdx.x >> lx, ny = kBlock >> lx;
    const uint32_t group = ((block_index() % tiles_x) << lx) + x;
    const uint64_t col = 8ull * group;
    const int columns = col >= a.dim ? 0 : a.dim - col < 8 ? static_cast<int>(a.dim - col) : 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    counts[wave][lane] = 0;

    // a wave's part of the ids: a run of whole steps of 64, in registers for both readings
    const uint32_t steps = (a.tokens + kBlock - 1) / kBlock, first = wave * steps;
    uint32_t row[kSteps];   // of the workgroup's; others are larger
    {
        Id raw[kSteps];
#pragma unroll
        for (int j = 0; j < kSteps; ++j) {
            const uint32_t t = 64 * (first + j) + lane;
            raw[j] = ~Id(0);
            if (static_cast<uint32_t>(j) < steps && t < a.tokens) raw[j] = static_cast<const Id *>(a.ids)[t];
        }
#pragma unroll
        for (int j = 0; j < kSteps; ++j)
            row[j] = raw[j] < a.vocab ? static_cast<uint32_t>(raw[j]) - v0 : 0xffffffffu;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSteps; ++j)
        if (row[j] < kSmallRows) atomicAdd(&counts[wave][row[j]], 1u);
    __syncthreads();
    if (wave == 0) {   // lane l: row l; where each wave's tokens of it begin
        uint32_t c[kSmallWaves], all = 0;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) {
            c[w] = counts[w][lane];
            all += c[w];
        }
        uint32_t sum = all;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t z = __shfl_up(sum, d);
            if (lane >= d) sum += z;
        }
        uint32_t at = sum - all;
        begins[lane] = at;
        if (lane == 63) begins[64] = sum;
        const uint64_t shared = __ballot(all > kSmallAlone);
        if (lane == 0) shared_rows = shared;
#pragma unroll
        for (int w = 0; w < kSmallWaves; ++w) {
            counts[w][lane] = at;
            at += c[w];
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
        uint64_t todo = __ballot(row[j] < kSmallRows);
        while (todo) {   // one row after the other: all its lanes at once
            const int f = __ffsll(static_cast<unsigned long long>(todo)) - 1;
            const uint32_t one = __builtin_amdgcn_readlane(row[j], f);
            const uint64_t lanes = todo & __ballot(row[j] == one);
            const uint32_t at = counts[wave][one];
            if (lanes >> lane & 1)
                list[at + __popcll(lanes & ((1ull << lane) - 1))] = 64 * (first + j) + lane;
            counts[wave][one] = at + __popcll(lanes);   // all lanes alike
            todo &= ~lanes;
        }
    }
    __syncthreads();

    const uint32_t rows = min(kSmallRows, a.vocab - v0);
    if (columns != 0) {
        for (uint32_t r = y; r < rows; r += ny) {
            const uint32_t from = begins[r], count = begins[r + 1] - from;
            if (count > kSmallAlone || (count == 0 && a.accumulate)) continue;
            float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            add_tokens<G, DROP>(sum, a, list + from, count, group, columns);
            write_row<OUT>(a, sum, count, v0 + r, group, columns);
        }
    }
    for (uint64_t todo = shared_rows; todo != 0; todo &= todo - 1) {   // the same for the whole workgroup
        const uint32_t r = __ffsll(static_cast<unsigned long long>(todo)) - 1;
        const uint32_t begin = begins[r], count = begins[r + 1] - begin;
        const uint32_t each = (count + ny - 1) / ny;
        const uint32_t from = min(y * each, count), to = min(from + each, count);
        float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if (columns != 0) add_tokens<G, DROP>(sum, a, list + begin + from, to - from, group, columns);
#pragma unroll
        for (int e = 0; e < 8; ++e) runs[threadIdx.x][e] = sum[e];
        __syncthreads();
        if (y == 0 && columns != 0) {
            const uint32_t used = (count + each - 1) / each;
            for (uint32_t i = 1; i < used; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum[e] += runs[(i << lx) + x][e];
            write_row<OUT>(a, sum, count, v0 + r, group, columns);
        }
        __syncthreads();
    }
}

template <int IDT, int G, int OUT>
hipError_t launch_few(const GradArgs &a, hipStream_t s) {
    const uint64_t groups = (a.dim + 7) / 8;
    int lx = 0;
    while (lx < 4 && (1ull << lx) < groups) ++lx;
    const uint32_t tiles_x = static_cast<uint32_t>((groups + (1ull << lx) - 1) >> lx);
    const uint64_t blocks = (static_cast<uint64_t>(a.vocab) + kSmallRows - 1) / kSmallRows * tiles_x;
    dim3 grid;
    if (!grid_of(blocks, kBlock, &grid)) return hipErrorInvalidConfiguration;
    if (a.drop.drop != 0) sum_few<IDT, G, OUT, true><<<grid, kBlock, 0, s>>>(a, lx, tiles_x);
    else sum_few<IDT, G, OUT, false><<<grid, kBlock, 0, s>>>(a, lx, tiles_x);
    return hipGetLastError();
}

template <int IDT>
hipError_t launch_few_typed(const GradArgs &a, int grad_dtype, int out_dtype, hipStream_t s) {
    if (grad_dtype == PS_F32)
        return out_dtype == PS_F32 ? launch_few<IDT, PS_F32, PS_F32>(a, s)
                                   : launch_few<IDT, PS_F32, PS_BF16>(a, s);
    return out_dtype == PS_F32 ? launch_few<IDT, PS_BF16, PS_F32>(a, s)
                               : launch_few<IDT, PS_BF16, PS_BF16>(a, s);
}

// Every workgroup reads all ids, and rows with many tokens are taken one after the other. In us,
// with dropout, in one launch and in three: 1824 tokens of 100 columns into 50000 rows 15 and 23,
// 2048 of 512 into 30000 21 and 27, 4096 of 1024 into 30000 34 and 36; but of 4096 into 30000 174
// and 102, and 4096 of 64 into 1000 36 and 18. These are ids whose numbers say nothing of how frequent
// they are: the sizes do not tell the host of others. Where the first rows are the most frequent, which
// one workgroup then has, the first takes 104 and 22, the third 141 and 36.
bool few(int64_t tokens, int64_t vocab, int64_t dim) {
    return tokens <= int64_t(kSmallTokens) && tokens <= vocab && dim <= 1024;
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
    const bool past = static_cast<uint64_t>(a.vocab) * a.dim * kBytes<OUT> > kCached;
    dim3 grid;
    if (!grid_of(blocks, kBlock, &grid)) return hipErrorInvalidConfiguration;
    const uint32_t pb = static_cast<uint32_t>(piece_blocks);
    if (a.drop.drop != 0) sum_rows<G, OUT, true><<<grid, kBlock, 0, s>>>(a, p, lx, tiles_x, pb, past);
    else sum_rows<G, OUT, false><<<grid, kBlock, 0, s>>>(a, p, lx, tiles_x, pb, past);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.pieces == 0) return e;
    const int join_lx = std::min(lx, kJoinMostGroups);
    const uint32_t join_x = static_cast<uint32_t>((groups + (1ull << join_lx) - 1) >> join_lx);
    const uint32_t join_blocks = (p.pieces + kJoinSlots - 1) / kJoinSlots * join_x;
    join_pieces<OUT><<<join_blocks, kBlock, 0, s>>>(a, p, join_lx, join_x);
    return hipGetLastError();
}

template <int IDT>
void launch_sort(const GradArgs &a, const Plan &p, Row *rows, uint32_t *perm, Piece *pieces, hipStream_t s) {
    // More waves share the ids of a workgroup, and take longer to start and to be brought together:
    // in us, with four waves and with sixteen, calls of 100 columns into 50000 rows in three launches, 2048
    // ids 21.1 and 22.4, 4096 26.7 and 26.4, 8192 30.8 and 28.4.
    const uint32_t n = a.tokens, v = a.vocab;
    if (n <= 4096) sort_tokens<IDT, 4, true><<<p.classes, 256, 0, s>>>(a.ids, n, v, p, rows, perm, pieces);
    else if (n <= kNoted)
        sort_tokens<IDT, 16, true><<<p.classes, 1024, 0, s>>>(a.ids, n, v, p, rows, perm, pieces);
    else sort_tokens<IDT, 16, false><<<p.classes, 1024, 0, s>>>(a.ids, n, v, p, rows, perm, pieces);
}

}  // namespace

size_t grad_workspace(int64_t tokens, int64_t vocab, int64_t dim) {
    if (few(tokens, vocab, dim)) return 0;
    return make_plan(tokens, vocab, dim).bytes;
}

hipError_t launch_grad(const GradArgs &a, int id_type, int grad_dtype, int out_dtype,
                       hipStream_t s) {
    if (few(a.tokens, a.vocab, static_cast<int64_t>(a.dim)))
        return id_type == PL_I32 ? launch_few_typed<PL_I32>(a, grad_dtype, out_dtype, s)
                                 : launch_few_typed<PL_I64>(a, grad_dtype, out_dtype, s);
    const Plan p = make_plan(a.tokens, a.vocab, static_cast<int64_t>(a.dim));
    char *ws = static_cast<char *>(a.workspace);
    Row *rows = reinterpret_cast<Row *>(ws + p.rows_at);
    uint32_t *perm = reinterpret_cast<uint32_t *>(ws + p.perm_at);
    Piece *pieces = reinterpret_cast<Piece *>(ws + p.pieces_at);
    if (id_type == PL_I32) launch_sort<PL_I32>(a, p, rows, perm, pieces, s);
    else launch_sort<PL_I64>(a, p, rows, perm, pieces, s);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (grad_dtype == PS_F32)
        return out_dtype == PS_F32 ? launch_sums<PS_F32, PS_F32>(a, p, s)
                                   : launch_sums<PS_F32, PS_BF16>(a, p, s);
    return out_dtype == PS_F32 ? launch_sums<PS_BF16, PS_F32>(a, p, s)
                               : launch_sums<PS_BF16, PS_BF16>(a, p, s);
}

}  // namespace gadei::learner
