// The norms after and before a block, with the block's gate and the stream's scale between them, and
// their gradients.
//
// Mathematics, of each row (N(v) = v r, r = (mean(v^2) + eps)^-1/2):
//
//   b = after * N(y) (or y)      h = scale x + gate * b      z = before * N(h)
//
// and from the gradients dh and dz, with u = dz * before and C columns:
//
//   dH = dh + rh (u - h rh^2 sum(u h) / C)            dx = scale dH      dbefore = sum over rows dz h rh
//   v = dH * gate * after                             dy = ry (v - y ry^2 sum(v y) / C)
//   dafter = sum over rows dH gate y ry               dgate = sum over its rows dH b
//
// sum(v y) is that of (dh + rh u - rh^3 sum(u h) / C h) gate after y: all sums of a row are taken in
// one reduction, without dH.
//
// Bound by memory. A row stays in registers, eight neighbouring columns a thread (`N` times), so each
// matrix is read and written once; longer rows are read again. Sums over rows stay in registers over
// a worker's rows, go to the workspace and are joined in order. Forward 16384 x 8192 bf16 takes 200 us
// (1.07 GB, 5.4 TB/s; a kernel that only adds takes 198), 4096 x 4096 with an fp32 stream 40 us (0.20 GB,
// 5.0), backward 16384 x 4096 bf16 with 32 gates 166 us and 7 for joining (0.81 GB, 4.9; vector
// instructions 60% of the time; a kernel that only adds takes 154). The loads of two or three rows ahead instead
// of one, or twice the workers, take as long.
//
// Rows that no thread's eights hold are read again for each sum: 4096 x 25088 bf16 245 us forward (0.82 GB, 3.4
// TB/s), 448 backward (1.23 GB, 2.8). Narrow ones leave lanes idle, as a wave or a workgroup has one row: 2^20 x 5
// fp32 857 and 2746 us (0.1 and 0.05 TB/s), 32768 x 100 bf16 19 and 58, 100000 x 188 51 and 145, backward as long as
// 100000 x 512 (71 and 143).
#include <algorithm>
#include <type_traits>

#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kJoinCols = 32;   // of a workgroup of `join`
constexpr int kGateRows = 4;    // threads that add up a column of a gate of few workers
constexpr int kSums = 6;
constexpr uint64_t kRowCols = 8 * 1024;        // of a row that 1024 threads hold, eight columns each

// Where a row begins; the same for all lanes of a wave, so that a lane's address is a 32-bit offset.
template <int DT>
__device__ __forceinline__ const void *row_of(const void *p, uint32_t row, int64_t ld) {
    return static_cast<const char *>(p) + static_cast<int64_t>(row) * ld * kBytes<DT>;
}
template <int DT>
__device__ __forceinline__ void *row_of(void *p, uint32_t row, int64_t ld) {
    return static_cast<char *>(p) + static_cast<int64_t>(row) * ld * kBytes<DT>;
}

// The wave's threadIdx.y.
__device__ __forceinline__ uint32_t wave_y() { return __builtin_amdgcn_readfirstlane(threadIdx.y); }

// A lane's column, which the compiler takes for another one each time: it would keep a 64-bit address a lane
// for every matrix, where a row's address and 32 bits a lane do.
__device__ __forceinline__ uint32_t now(uint32_t col) {
    asm volatile("" : "+v"(col));
    return col;
}

// Eight columns as loaded: zeros past `count`. EIGHTS: all of them or none.
template <int DT, bool EIGHTS>
__device__ __forceinline__ Bits8<DT> bits8(const void *p, uint32_t at, int count) {
    if (count == 8) return load8<DT>(p, at);
    if constexpr (EIGHTS) return Bits8<DT>{};
    else return load8_some<DT>(p, at, count);
}

// Of a vector of weights, or ones where there is none.
template <bool EIGHTS>
__device__ __forceinline__ void vector8(float (&w)[8], const void *p, int bf16, uint32_t at, int count) {
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    } else if (bf16) {
        widen8<PS_BF16>(w, bits8<PS_BF16, EIGHTS>(p, at, count));
    } else {
        widen8<PS_F32>(w, bits8<PS_F32, EIGHTS>(p, at, count));
    }
}

// The same bits, which the compiler takes for others: it would keep what it has widened of them through
// a row's reduction, in twice the registers.
__device__ __forceinline__ void anew(Bits8<PS_BF16> &x) { asm volatile("" : "+v"(x.a)); }
__device__ __forceinline__ void anew(Bits8<PS_F32> &) {}

template <int DT>
__device__ __forceinline__ void row8(float (&x)[8], const void *p, uint32_t at, int count) {
    widen8<DT>(x, bits8<DT, false>(p, at, count));
}

template <int DT>
__device__ __forceinline__ void put8(void *p, uint32_t at, const float (&x)[8], int count) {
    if (count == 8) store8<DT>(p, at, x);
    else store_some<DT>(p, at, x, count);
}

// Results of a row. They stay in the caches, as far as there is room, for the layer that reads them: stores past
// those save less than that (16384 x 8192 bf16 212 us with either, 4096 x 4096 28 and 23).
template <int DT, bool EIGHTS>
__device__ __forceinline__ void put_row8(void *p, uint32_t at, const float (&x)[8], int count) {
    if (count == 0) return;
    if constexpr (EIGHTS) store8<DT>(p, at, x);
    else put8<DT>(p, at, x, count);
}

__device__ __forceinline__ int count_at(uint64_t cols, uint64_t col) {
    return cols >= col + 8 ? 8 : cols > col ? static_cast<int>(cols - col) : 0;
}

// A thread's eight columns of a row of at least as many, all or none of them. The row's last thread goes back to
// where there are eight: its first `twice` are its neighbour's too. It leaves them out of sums over the row;
// their results are the same bits from both. ODD: the row's columns are not eights.
struct Place {
    uint32_t col;
    int count, twice;
    template <bool ODD>
    __device__ __forceinline__ static Place of(uint32_t thread, uint64_t cols) {
        const uint32_t col = 8 * thread, n = static_cast<uint32_t>(cols);
        const bool in = col < n;
        if constexpr (!ODD) return Place{col, in ? 8 : 0, 0};
        const uint32_t from = in ? min(col, n - 8) : col;
        return Place{from, in ? 8 : 0, static_cast<int>(col - from)};
    }
};

template <bool ODD>
__device__ __forceinline__ void leave_out(float (&x)[8], int twice) {
    if constexpr (ODD) {
#pragma unroll
        for (int e = 0; e < 7; ++e) x[e] = e < twice ? 0.0f : x[e];
    }
}

// Sums over the sixteen lanes of a row of lanes, in all of them.
__device__ __forceinline__ float sum16(float x) {
    auto rotated = [](float v, auto by) {
        constexpr int kRotate = 0x120 + decltype(by)::value;
        return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), kRotate, 0xf, 0xf, true));
    };
    x += rotated(x, std::integral_constant<int, 8>());
    x += rotated(x, std::integral_constant<int, 4>());
    x += rotated(x, std::integral_constant<int, 2>());
    x += rotated(x, std::integral_constant<int, 1>());
    return x;
}

__device__ __forceinline__ float sum64(float x) {
    x = sum16(x);
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    const auto q = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}

// Sums over the threads of a row: a wave, or a whole workgroup, whose waves' sums go through `lds`
// (two places in turn, so that one barrier is enough). There, sixteen lanes add up each sum.
template <int K>
__device__ __forceinline__ void sum_row(float (&s)[K], float *lds, int *turn) {
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = sum64(s[k]);
    const int waves = static_cast<int>(blockDim.x) >> 6, lane = static_cast<int>(threadIdx.x) & 63;
    if (waves == 1) return;
    float *at = lds + *turn * 16 * kSums;
    *turn ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) at[16 * k + (threadIdx.x >> 6)] = s[k];
    }
    __syncthreads();
    const int wave = lane & 15, first = lane >> 4;
#pragma unroll
    for (int k0 = 0; k0 < K; k0 += 4) {
        const float v = sum16(wave < waves && k0 + first < K ? at[16 * (k0 + first) + wave] : 0.0f);
#pragma unroll
        for (int k = k0; k < K && k < k0 + 4; ++k)
            s[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 16 * (k - k0)));
    }
}

__device__ __forceinline__ float inverse_root(float sum, uint64_t cols, float eps) {
    return 1.0f / sqrtf(sum / static_cast<float>(cols) + eps);
}

// ----------------------------------------------------------------- forward

__device__ __forceinline__ void times8(float (&a)[8], const float (&b)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] *= b[e];
}

// The row of the gate that is row `row`'s.
template <bool EIGHTS, class Args>
__device__ __forceinline__ void gate8(float (&w)[8], const Args &a, uint32_t row, uint32_t col, int count) {
    const void *const gate = a.gate_bf16 ? row_of<PS_BF16>(a.gate, row / a.per_gate, a.gate_ld)
                                         : row_of<PS_F32>(a.gate, row / a.per_gate, a.gate_ld);
    vector8<EIGHTS>(w, a.gate == nullptr ? nullptr : gate, a.gate_bf16, col, count);
}

// after * gate.
template <bool EIGHTS, class Args>
__device__ __forceinline__ void branch_scale(float (&w)[8], const Args &a, uint32_t row, uint32_t col, int count) {
    float gate[8];
    vector8<EIGHTS>(w, a.after, a.weight_bf16, col, count);
    gate8<EIGHTS>(gate, a, row, col, count);
    times8(w, gate);
}

// What the block leaves in the stream: h of eight columns.
template <int X>
__device__ __forceinline__ void stream8(float (&h)[8], const NormArgs &a, const Bits8<X> &x_bits, const float (&y)[8],
                                        float ry, const float (&w)[8]) {
    float x[8];
    widen8<X>(x, x_bits);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = a.scale * x[e] + y[e] * ry * w[e];
}

// A worker, a wave or a workgroup, takes `rows_each` rows one after another, the next one's loads under
// way; the vectors stay in registers.
template <int X, int Y, int N, bool BLOCK, bool ODD>
__global__ __launch_bounds__(1024) void norm(NormArgs a, uint32_t rows_each) {
    constexpr bool EIGHTS = true;
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint64_t first = (static_cast<uint64_t>(block_index()) * blockDim.y + wave_y()) * rows_each;
    if (first >= a.rows) return;   // a whole wave, of those that no barrier waits for
    const uint32_t last = static_cast<uint32_t>(min(static_cast<uint64_t>(a.rows), first + rows_each));
    uint32_t col[N];
    int count[N], twice[N];
    float branch[N][8], before[N][8];
    Bits8<X> next_x[N];
    Bits8<Y> next_y[N];
    auto load = [&](uint32_t row) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            next_x[i] = bits8<X, EIGHTS>(row_of<X>(a.x, row, a.x_ld), now(col[i]), count[i]);
            if constexpr (BLOCK) next_y[i] = bits8<Y, EIGHTS>(row_of<Y>(a.y, row, a.y_ld), now(col[i]), count[i]);
        }
    };
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Place place = Place::of<ODD>(threadIdx.x + i * blockDim.x, a.cols);
        col[i] = place.col;
        count[i] = place.count;
        twice[i] = place.twice;
    }
    load(static_cast<uint32_t>(first));
#pragma unroll
    for (int i = 0; i < N; ++i) vector8<EIGHTS>(before[i], a.before, a.weight_bf16, col[i], count[i]);
    uint32_t gate_ends = static_cast<uint32_t>(first);
    for (uint32_t row = static_cast<uint32_t>(first); row < last; ++row) {
        if (BLOCK && row >= gate_ends) {
            // of all rows where there is no gate
            gate_ends = a.gate == nullptr ? a.rows : (row / a.per_gate + 1) * a.per_gate;
#pragma unroll
            for (int i = 0; i < N; ++i) branch_scale<EIGHTS>(branch[i], a, row, now(col[i]), count[i]);
        }
        float h[N][8];
        Bits8<X> x[N];
        Bits8<Y> y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = next_x[i];
            if constexpr (BLOCK) y[i] = next_y[i];
        }
        if (row + 1 < last) load(row + 1);
        float s[1] = {0.0f};
        if constexpr (BLOCK) {
            float ry = 1.0f;
            if (a.after != nullptr) {
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    float v[8];
                    widen8<Y>(v, y[i]);
                    leave_out<ODD>(v, twice[i]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[0] += v[e] * v[e];
                    anew(y[i]);
                }
                sum_row(s, lds, &turn);
                ry = inverse_root(s[0], a.cols, a.eps);
                s[0] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float v[8];
                widen8<Y>(v, y[i]);
                stream8<X>(h[i], a, x[i], v, ry, branch[i]);
                put_row8<X, EIGHTS>(row_of<X>(a.out, row, a.out_ld), now(col[i]), h[i], count[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) widen8<X>(h[i], x[i]);
        }
        if (a.normed == nullptr) continue;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += ODD && e < twice[i] ? 0.0f : h[i][e] * h[i][e];
        sum_row(s, lds, &turn);
        const float rh = inverse_root(s[0], a.cols, a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] *= rh * before[i][e];
            put_row8<Y, EIGHTS>(row_of<Y>(a.normed, row, a.normed_ld), now(col[i]), h[i], count[i]);
        }
    }
}

// Longer rows, and those of fewer than eight columns: a workgroup a row, which it reads again for each sum.
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(1024) void norm_long(NormArgs a) {
    constexpr bool EIGHTS = false;
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint32_t row = block_index();
    if (row >= a.rows) return;
    const uint32_t first = 8 * threadIdx.x, step = 8 * blockDim.x;
    float s[1] = {0.0f}, ry = 1.0f;
    if (BLOCK && a.after != nullptr) {
        for (uint32_t col = first; col < a.cols; col += step) {
            float y[8];
            row8<Y>(y, row_of<Y>(a.y, row, a.y_ld), col, count_at(a.cols, col));
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += y[e] * y[e];
        }
        sum_row(s, lds, &turn);
        ry = inverse_root(s[0], a.cols, a.eps);
        s[0] = 0.0f;
    }
    auto stream = [&](float (&h)[8], uint32_t col, int count) {
        if constexpr (BLOCK) {
            float y[8], w[8];
            row8<Y>(y, row_of<Y>(a.y, row, a.y_ld), col, count);
            branch_scale<EIGHTS>(w, a, row, col, count);
            stream8<X>(h, a, bits8<X, EIGHTS>(row_of<X>(a.x, row, a.x_ld), col, count), y, ry, w);
        } else {
            row8<X>(h, row_of<X>(a.x, row, a.x_ld), col, count);
        }
    };
    for (uint32_t col = first; col < a.cols; col += step) {
        const int count = count_at(a.cols, col);
        float h[8];
        stream(h, col, count);
        if (BLOCK) put8<X>(row_of<X>(a.out, row, a.out_ld), col, h, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += h[e] * h[e];
    }
    if (a.normed == nullptr) return;
    sum_row(s, lds, &turn);
    const float rh = inverse_root(s[0], a.cols, a.eps);
    for (uint32_t col = first; col < a.cols; col += step) {
        const int count = count_at(a.cols, col);
        float h[8], w[8];
        stream(h, col, count);
        vector8<EIGHTS>(w, a.before, a.weight_bf16, col, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] *= rh * w[e];
        put8<Y>(row_of<Y>(a.normed, row, a.normed_ld), col, h, count);
    }
}

// ---------------------------------------------------------------- backward

// Workers and their rows, in order; where their sums over rows are in the workspace.
struct Split {
    uint32_t workers, rows;   // of a worker
    uint64_t pitch;           // columns, padded to eights
    float *before, *after;    // [worker][pitch]
    float *gate;              // [worker][2][pitch]: of a gate that began before the worker's rows, and of one
                              // that begins in them and goes on
    f32x4 *rows_of;           // of rows that no worker holds: rh, k1, ry, k2 of each
};

// Eight columns of a row, as loaded.
template <int X, int Y, bool BLOCK, bool EIGHTS>
struct RowBits {
    Bits8<X> h, dh;
    Bits8<Y> y, dz;
    __device__ __forceinline__ void load(const NormGradArgs &a, uint32_t row, uint32_t col, int count) {
        // without dz nothing depends on h, an infinite one's products with zeros neither
        h = a.dz != nullptr ? bits8<X, EIGHTS>(row_of<X>(a.h, row, a.h_ld), col, count) : Bits8<X>{};
        if constexpr (BLOCK) y = bits8<Y, EIGHTS>(row_of<Y>(a.y, row, a.y_ld), col, count);
        dh = a.dh != nullptr ? bits8<X, EIGHTS>(row_of<X>(a.dh, row, a.dh_ld), col, count) : Bits8<X>{};
        dz = a.dz != nullptr ? bits8<Y, EIGHTS>(row_of<Y>(a.dz, row, a.dz_ld), col, count) : Bits8<Y>{};
    }
};

// What a thread keeps of its columns: the vectors, and sums over rows. In a gate's rows the gradients
// of the gate and of after share the sum of dH N(y), times after and times the gate.
struct Columns {
    float branch[8];                 // after * gate
    float d_before[8], d_branch[8];
    f32x4 *before, *d_after;         // in LDS, the thread's own: two fours each, `apart` from one another
    uint32_t apart;
};

// h h, u h; y y, and of p = gate after y: p dh, p u, p h
template <bool ODD, int X, int Y, bool BLOCK, bool EIGHTS>
__device__ __forceinline__ void add_sums(float (&s)[kSums], const RowBits<X, Y, BLOCK, EIGHTS> &v, const Columns &c,
                                         int twice) {
    float h[8], dz[8], y[8], dh[8];
    widen8<X>(h, v.h);
    widen8<Y>(dz, v.dz);
    if constexpr (BLOCK) {
        widen8<Y>(y, v.y);
        widen8<X>(dh, v.dh);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if (ODD && e < twice) continue;
        const float u = dz[e] * c.before[e / 4 * c.apart][e % 4];
        s[0] += h[e] * h[e];
        s[1] += u * h[e];
        if constexpr (BLOCK) {
            const float p = c.branch[e] * y[e];
            s[2] += y[e] * y[e];
            s[3] += p * dh[e];
            s[4] += p * u;
            s[5] += p * h[e];
        }
    }
}

// rh, k1 = rh^2 mean(u h), ry, k2 = ry^2 mean(v y). Without a norm before or after: 0, 0 and 1, 0. A factor's square
// by itself passes fp32's range in a row of zeros where eps is below 2^-128.
__device__ __forceinline__ f32x4 row_factors(const NormGradArgs &a, const float (&s)[kSums]) {
    const float n = static_cast<float>(a.cols);
    f32x4 r = {0.0f, 0.0f, 1.0f, 0.0f};
    if (a.dz != nullptr) {
        r[0] = inverse_root(s[0], a.cols, a.eps);
        r[1] = r[0] * (r[0] * (s[1] / n));
    }
    if (a.after != nullptr) {
        r[2] = inverse_root(s[2], a.cols, a.eps);
        r[3] = r[2] * (r[2] * ((s[3] + r[0] * (s[4] - r[1] * s[5])) / n));
    }
    return r;
}

template <int X, int Y, bool BLOCK, bool EIGHTS>
__device__ __forceinline__ void take_row(const NormGradArgs &a, const RowBits<X, Y, BLOCK, EIGHTS> &v, f32x4 r,
                                         uint32_t row, uint32_t col, int count, Columns &c) {
    float h[8], dz[8], d[8];
    widen8<X>(h, v.h);
    widen8<Y>(dz, v.dz);
    widen8<X>(d, v.dh);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        d[e] += r[0] * (dz[e] * c.before[e / 4 * c.apart][e % 4] - h[e] * r[1]);
        c.d_before[e] += dz[e] * (h[e] * r[0]);
        h[e] = a.scale * d[e];
    }
    put_row8<X, EIGHTS>(row_of<X>(a.dx, row, a.dx_ld), col, h, count);
    if constexpr (BLOCK) {
        float y[8];
        widen8<Y>(y, v.y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            c.d_branch[e] += d[e] * (y[e] * r[2]);
            d[e] *= c.branch[e];
        }
        if (a.after != nullptr) {   // else y has no part in it, and may be infinite
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = r[2] * (d[e] - y[e] * r[3]);
        }
        put_row8<Y, EIGHTS>(row_of<Y>(a.dy, row, a.dy_ld), col, d, count);
    }
}

// twice: of them, what the neighbour adds to what is there.
template <bool EIGHTS>
__device__ __forceinline__ void put_result(const NormGradArgs &a, void *p, uint32_t at, float (&x)[8], int count,
                                           int twice) {
    if (a.accumulate) {
        float old[8];
        vector8<EIGHTS>(old, p, a.out_bf16, at, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < twice || e >= count) continue;
            if (a.out_bf16) store1<PS_BF16>(p, at + e, old[e] + x[e]);
            else store1<PS_F32>(p, at + e, old[e] + x[e]);
        }
    } else if (a.out_bf16) {
        put8<PS_BF16>(p, at, x, count);
    } else {
        put8<PS_F32>(p, at, x, count);
    }
}

// The first of a gate's rows among the worker's (without a gate: of all rows); when they end.
template <bool EIGHTS>
__device__ __forceinline__ uint32_t begin_gate(const NormGradArgs &a, uint32_t row, uint32_t last, uint32_t col,
                                               int count, Columns &c) {
    branch_scale<EIGHTS>(c.branch, a, row, col, count);
#pragma unroll
    for (int e = 0; e < 8; ++e) c.d_branch[e] = 0.0f;
    return a.gate == nullptr ? last : min(last, (row / a.per_gate + 1) * a.per_gate);
}

// The last of them has been taken, before `end`.
template <bool EIGHTS>
__device__ __forceinline__ void end_gate(const NormGradArgs &a, const Split &sp, uint32_t worker, uint32_t first,
                                         uint32_t last, uint32_t end, uint32_t col, int count, int twice, Columns &c) {
    float w[8];
    if (a.dafter != nullptr) {
        gate8<EIGHTS>(w, a, end - 1, col, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) c.d_after[e / 4 * c.apart][e % 4] += w[e] * c.d_branch[e];
    }
    if (a.dgate == nullptr || count == 0) return;
    vector8<EIGHTS>(w, a.after, a.weight_bf16, col, count);
    times8(c.d_branch, w);
    const uint32_t gate = (end - 1) / a.per_gate;
    const uint64_t begins = static_cast<uint64_t>(gate) * a.per_gate, ends = begins + a.per_gate;
    if (begins >= first && ends <= last) {
        void *const to = a.out_bf16 ? row_of<PS_BF16>(a.dgate, gate, a.dgate_ld)
                                    : row_of<PS_F32>(a.dgate, gate, a.dgate_ld);
        put_result<EIGHTS>(a, to, col, c.d_branch, count, twice);
    } else {
        const uint64_t slot = 2 * static_cast<uint64_t>(worker) + (begins >= first ? 1 : 0);
        store8<PS_F32>(sp.gate + slot * sp.pitch, col, c.d_branch);
    }
}

template <bool EIGHTS>
__device__ __forceinline__ void begin_worker(const NormGradArgs &a, uint32_t col, int count, Columns &c) {
    float w[8];
    vector8<EIGHTS>(w, a.before, a.weight_bf16, col, count);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        c.before[e / 4 * c.apart][e % 4] = w[e];
        c.branch[e] = c.d_before[e] = c.d_branch[e] = 0.0f;
    }
    c.d_after[0] = c.d_after[c.apart] = f32x4{0, 0, 0, 0};
}

__device__ __forceinline__ void end_worker(const NormGradArgs &a, const Split &sp, uint32_t worker, uint32_t col,
                                           int count, const Columns &c) {
    if (count == 0) return;
    const uint64_t at = worker * sp.pitch;
    if (a.dbefore != nullptr) store8<PS_F32>(sp.before + at, col, c.d_before);
    if (a.dafter == nullptr) return;
    const f32x4 x = c.d_after[0], y = c.d_after[c.apart];
    const float sum[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
    store8<PS_F32>(sp.after + at, col, sum);
}

// A worker is a wave or a workgroup; it takes its rows one after another, the next one's loads under way.
template <int X, int Y, bool BLOCK, bool ODD>
__global__ __launch_bounds__(1024, 4) void norm_grad(NormGradArgs a, Split sp) {
    constexpr bool EIGHTS = true;
    __shared__ float lds[2 * 16 * kSums];
    extern __shared__ f32x4 own[];   // four a thread
    int turn = 0;
    const uint32_t worker = block_index() * blockDim.y + wave_y();
    if (worker >= sp.workers) return;   // a whole wave, of those that no barrier waits for
    const uint32_t first = worker * sp.rows, last = min(a.rows - first, sp.rows) + first;
    const Place place = Place::of<ODD>(threadIdx.x, a.cols);
    const uint32_t col = place.col;
    const int count = place.count, twice = place.twice;
    RowBits<X, Y, BLOCK, EIGHTS> next;
    next.load(a, first, col, count);
    Columns c;
    c.apart = blockDim.x * blockDim.y;
    c.before = own + threadIdx.y * blockDim.x + threadIdx.x;
    c.d_after = c.before + 2 * c.apart;
    begin_worker<EIGHTS>(a, col, count, c);
    for (uint32_t row = first; row < last;) {
        const uint32_t end = BLOCK ? begin_gate<EIGHTS>(a, row, last, now(col), count, c) : last;
        for (; row < end; ++row) {
            RowBits<X, Y, BLOCK, EIGHTS> v = next;
            if (row + 1 < last) next.load(a, row + 1, now(col), count);
            float s[kSums] = {};
            add_sums<ODD>(s, v, c, twice);
            sum_row(s, lds, &turn);
            anew(v.h);
            anew(v.dh);
            anew(v.dz);
            if constexpr (BLOCK) anew(v.y);
            take_row(a, v, row_factors(a, s), row, now(col), count, c);
        }
        if constexpr (BLOCK) end_gate<EIGHTS>(a, sp, worker, first, last, end, now(col), count, twice, c);
    }
    end_worker(a, sp, worker, col, count, c);
}

// Longer rows, and those of fewer than eight columns: first their sums, a workgroup a row, ...
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(1024) void row_sums(NormGradArgs a, Split sp) {
    constexpr bool EIGHTS = false;
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint32_t row = block_index();
    if (row >= a.rows) return;
    float s[kSums] = {};
    for (uint32_t col = 8 * threadIdx.x; col < a.cols; col += 8 * blockDim.x) {
        const int count = count_at(a.cols, col);
        RowBits<X, Y, BLOCK, EIGHTS> v;
        v.load(a, row, col, count);
        Columns c;
        float w[8];
        vector8<EIGHTS>(w, a.before, a.weight_bf16, col, count);
        f32x4 before[2] = {{w[0], w[1], w[2], w[3]}, {w[4], w[5], w[6], w[7]}};
        c.before = before;
        c.apart = 1;
        if constexpr (BLOCK) branch_scale<EIGHTS>(c.branch, a, row, col, count);
        add_sums<false>(s, v, c, 0);
    }
    sum_row(s, lds, &turn);
    if (threadIdx.x == 0) sp.rows_of[row] = row_factors(a, s);
}

// ... then strips of columns.
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(256) void norm_grad_long(NormGradArgs a, Split sp, uint32_t strips) {
    constexpr bool EIGHTS = false;
    __shared__ f32x4 own[4 * 256];
    const uint64_t worker64 = block_index() / strips;
    if (worker64 >= sp.workers) return;
    const uint32_t worker = static_cast<uint32_t>(worker64);
    const uint32_t first = worker * sp.rows, last = min(a.rows - first, sp.rows) + first;
    const uint32_t col = 8 * (threadIdx.x + 256 * (block_index() % strips));
    const int count = count_at(a.cols, col);
    Columns c;
    c.apart = 256;
    c.before = own + threadIdx.x;
    c.d_after = c.before + 2 * c.apart;
    begin_worker<EIGHTS>(a, col, count, c);
    for (uint32_t row = first; row < last;) {
        const uint32_t end = BLOCK ? begin_gate<EIGHTS>(a, row, last, now(col), count, c) : last;
        for (; row < end; ++row) {
            RowBits<X, Y, BLOCK, EIGHTS> v;
            v.load(a, row, now(col), count);
            take_row(a, v, sp.rows_of[row], row, now(col), count, c);
        }
        if constexpr (BLOCK) end_gate<EIGHTS>(a, sp, worker, first, last, end, now(col), count, 0, c);
    }
    end_worker(a, sp, worker, col, count, c);
}

// The workers' sums, in order: y = 0 and 1 dbefore and dafter, by all threads of a column; from 2 on the gates
// whose rows are more than one worker's, by as many or, `short_gates`, kGateRows threads of a column each: of a
// few gates gate i, else the one that goes from worker i into the next.
template <int ROWS>
__global__ __launch_bounds__(kJoinCols * ROWS) void join(NormGradArgs a, Split sp, bool few_gates, uint32_t gates,
                                                       bool short_gates) {
    __shared__ float lds[ROWS][kJoinCols];
    const int x = threadIdx.x;
    const bool vector = blockIdx.y < 2, whole = vector || !short_gates;
    const uint32_t y = threadIdx.y & ((whole ? ROWS : kGateRows) - 1);
    const uint64_t col = static_cast<uint64_t>(blockIdx.x) * kJoinCols + x;
    void *const out = blockIdx.y == 0 ? a.dbefore : blockIdx.y == 1 ? a.dafter : a.dgate;
    if (out == nullptr) return;
    int64_t at = static_cast<int64_t>(col);
    uint32_t from = 0, to = sp.workers;
    const float *p = blockIdx.y == 0 ? sp.before : sp.after;
    uint64_t pitch = sp.pitch;
    bool mine = col < a.cols;
    float v = 0.0f;
    if (!vector) {
        const uint64_t i = whole ? blockIdx.y - 2 : (blockIdx.y - 2) * (ROWS / kGateRows) + threadIdx.y / kGateRows;
        const uint64_t boundary = (i + 1) * sp.rows;
        const uint64_t gate = few_gates ? i : boundary / a.per_gate;
        const uint64_t begins = gate * a.per_gate, ends = begins + a.per_gate;
        // not: no gate crosses this boundary, or it does not begin in this worker's rows
        mine = mine && i < gates && (few_gates || (begins != boundary && begins + sp.rows >= boundary));
        from = static_cast<uint32_t>(begins / sp.rows);
        to = static_cast<uint32_t>((ends - 1) / sp.rows) + 1;
        mine = mine && to > from + 1;
        at += static_cast<int64_t>(gate) * a.dgate_ld;
        p = sp.gate;
        pitch = 2 * sp.pitch;
        if (mine && y == 0) v = p[(2ull * from + 1) * sp.pitch + col];
        ++from;
    }
    auto add = [&](auto step) {
#pragma unroll 8
        for (uint32_t w = from + y; w < to; w += decltype(step)::value) v += p[w * pitch + col];
    };
    if (mine && whole) add(std::integral_constant<uint32_t, ROWS>());
    else if (mine) add(std::integral_constant<uint32_t, kGateRows>());
    lds[threadIdx.y][x] = v;
    __syncthreads();
    if (y != 0 || !mine) return;
    v = 0.0f;
    if (whole) {
#pragma unroll
        for (int i = 0; i < ROWS; ++i) v += lds[i][x];
    } else {
#pragma unroll
        for (int i = 0; i < kGateRows; ++i) v += lds[threadIdx.y + i][x];
    }
    if (a.accumulate) v += a.out_bf16 ? load1<PS_BF16>(out, at) : load1<PS_F32>(out, at);
    if (a.out_bf16) store1<PS_BF16>(out, at, v);
    else store1<PS_F32>(out, at, v);
}

// A gate's gradient from no rows.
__global__ __launch_bounds__(256) void no_rows(NormGradArgs a) {
    const uint64_t i = static_cast<uint64_t>(block_index()) * 256 + threadIdx.x;
    if (i >= a.gates * a.cols) return;
    const int64_t at = static_cast<int64_t>(i / a.cols) * a.dgate_ld + static_cast<int64_t>(i % a.cols);
    if (a.out_bf16) store1<PS_BF16>(a.dgate, at, 0.0f);
    else store1<PS_F32>(a.dgate, at, 0.0f);
}

// --------------------------------------------------------------- launches

// Threads of a row of so many columns, eight a thread: whole waves.
uint32_t threads_of(uint64_t cols) { return static_cast<uint32_t>(64 * std::min<uint64_t>(16, (cols + 511) / 512)); }

template <int X, int Y, bool BLOCK>
hipError_t launch(const NormArgs &a, hipStream_t s) {
    const uint32_t threads = threads_of(a.cols);
    const uint32_t together = threads == 64 ? 4 : 1;   // workers of a workgroup
    dim3 grid;
    if (a.cols < 8 || a.cols > 2 * kRowCols) {
        if (!grid_of(a.rows, threads, &grid)) return hipErrorInvalidConfiguration;
        norm_long<X, Y, BLOCK><<<grid, threads, 0, s>>>(a);
        return hipGetLastError();
    }
    // In us, with one row a worker, with as many workers as the card has room for, and with 4096: 16384 x
    // 8192 bf16 246, 215 and 195, without a gate 208, 216 and 197; 16384 x 5000 190, 166 and 148; but rows
    // of a wave, 200000 x 512, 139, 168 and 170.
    const uint64_t most = threads == 64 ? ~uint64_t(0) >> 1 : 4096;
    const uint32_t each = static_cast<uint32_t>((a.rows + most - 1) / most);
    const uint64_t workers = (a.rows + each - 1ull) / each;
    if (!grid_of((workers + together - 1) / together, threads * together, &grid)) return hipErrorInvalidConfiguration;
    const dim3 block(threads, together);
    const bool odd = a.cols % 8 != 0;
    if (a.cols > kRowCols && odd) norm<X, Y, 2, BLOCK, true><<<grid, block, 0, s>>>(a, each);
    else if (a.cols > kRowCols) norm<X, Y, 2, BLOCK, false><<<grid, block, 0, s>>>(a, each);
    else if (odd) norm<X, Y, 1, BLOCK, true><<<grid, block, 0, s>>>(a, each);
    else norm<X, Y, 1, BLOCK, false><<<grid, block, 0, s>>>(a, each);
    return hipGetLastError();
}

template <int X>
hipError_t launch(const NormArgs &a, int y_dtype, hipStream_t s) {
    if (a.y == nullptr)
        return y_dtype == PS_F32 ? launch<X, PS_F32, false>(a, s) : launch<X, PS_BF16, false>(a, s);
    return y_dtype == PS_F32 ? launch<X, PS_F32, true>(a, s) : launch<X, PS_BF16, true>(a, s);
}

// Backward: whether workers hold whole rows.
bool in_registers(uint64_t cols) { return cols >= 8 && cols <= kRowCols; }

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

Split split(uint64_t rows, uint64_t cols) {
    Split sp{};
    sp.pitch = (cols + 7) & ~uint64_t(7);
    if (rows == 0) return sp;
    // In us with 256, 512, 1024 and 2048 workers, their sums' joining included: 16384 x 4096 bf16 166, 175,
    // 187 and 198; 32768 x 1024 165, 122, 95 and 110; 100000 x 512 392, 209, 137 and 148
    const uint64_t most = in_registers(cols) ? std::clamp<uint64_t>(2048 * 64 / threads_of(cols), 256, 1024)
                                             : std::clamp<uint64_t>(1024 * 2048 / cols, 64, 1024);
    sp.rows = static_cast<uint32_t>((rows + most - 1) / most);
    sp.workers = static_cast<uint32_t>((rows + sp.rows - 1) / sp.rows);
    return sp;
}

template <int X, int Y, bool BLOCK>
hipError_t launch(const NormGradArgs &a, hipStream_t s) {
    Split sp = split(a.rows, a.cols);
    const size_t each = align256(sizeof(float) * sp.workers * sp.pitch);
    char *ws = static_cast<char *>(a.workspace);
    sp.before = reinterpret_cast<float *>(ws);
    sp.after = reinterpret_cast<float *>(ws + each);
    sp.gate = reinterpret_cast<float *>(ws + 2 * each);
    sp.rows_of = reinterpret_cast<f32x4 *>(ws + 4 * each);
    const uint32_t threads = threads_of(a.cols);
    dim3 grid;
    if (a.rows == 0) {
        if (a.accumulate) return hipSuccess;
        if (a.dgate != nullptr) {
            if (!grid_of((a.gates * a.cols + 255) / 256, 256, &grid)) return hipErrorInvalidConfiguration;
            no_rows<<<grid, 256, 0, s>>>(a);
        }
    } else if (in_registers(a.cols)) {
        const uint32_t together = threads == 64 ? 4 : 1;
        grid = dim3((sp.workers + together - 1) / together);
        const dim3 block(threads, together);
        const uint32_t own = 4 * sizeof(f32x4) * threads * together;
        if (a.cols % 8 != 0) norm_grad<X, Y, BLOCK, true><<<grid, block, own, s>>>(a, sp);
        else norm_grad<X, Y, BLOCK, false><<<grid, block, own, s>>>(a, sp);
    } else {
        if (!grid_of(a.rows, threads, &grid)) return hipErrorInvalidConfiguration;
        row_sums<X, Y, BLOCK><<<grid, threads, 0, s>>>(a, sp);
        const uint64_t strips = (a.cols + 2047) / 2048;
        if (!grid_of(strips * sp.workers, 256, &grid)) return hipErrorInvalidConfiguration;
        norm_grad_long<X, Y, BLOCK><<<grid, 256, 0, s>>>(a, sp, static_cast<uint32_t>(strips));
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const bool gates = a.dgate != nullptr && a.rows != 0 && sp.rows % a.per_gate != 0;
    if (a.dbefore == nullptr && a.dafter == nullptr && !gates) return hipSuccess;
    const bool few_gates = a.gates < sp.workers, many = sp.workers > 64;
    const uint32_t crossing = !gates ? 0 : few_gates ? a.gates : sp.workers - 1;
    // Of 32 gates of 8 workers each, 16384 x 4096 bf16 in all 176 us with short ones and 185 without, of 16 gates,
    // 2048 x 16384, 155 and 176, of 100, 16000 x 4096, 177 and 210.
    const bool short_gates = a.per_gate <= 32ull * sp.rows;
    const uint32_t rows_y = many ? 32 : 4, together = short_gates ? rows_y / kGateRows : 1;
    grid = dim3(static_cast<uint32_t>((a.cols + kJoinCols - 1) / kJoinCols), 2 + (crossing + together - 1) / together);
    if (many) join<32><<<grid, dim3(kJoinCols, 32), 0, s>>>(a, sp, few_gates, crossing, short_gates);
    else join<4><<<grid, dim3(kJoinCols, 4), 0, s>>>(a, sp, few_gates, crossing, short_gates);
    return hipGetLastError();
}

template <int X>
hipError_t launch(const NormGradArgs &a, int y_dtype, hipStream_t s) {
    if (a.y == nullptr)
        return y_dtype == PS_F32 ? launch<X, PS_F32, false>(a, s) : launch<X, PS_BF16, false>(a, s);
    return y_dtype == PS_F32 ? launch<X, PS_F32, true>(a, s) : launch<X, PS_BF16, true>(a, s);
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, int x_dtype, int y_dtype, hipStream_t s) {
    return x_dtype == PS_F32 ? launch<PS_F32>(a, y_dtype, s) : launch<PS_BF16>(a, y_dtype, s);
}

size_t norm_grad_workspace(int64_t rows, int64_t cols) {
    const Split sp = split(rows, cols);
    return 4 * align256(sizeof(float) * sp.workers * sp.pitch) +
           (!in_registers(static_cast<uint64_t>(cols)) ? sizeof(f32x4) * static_cast<size_t>(rows) : 0);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int x_dtype, int y_dtype, hipStream_t s) {
    return x_dtype == PS_F32 ? launch<PS_F32>(a, y_dtype, s) : launch<PS_BF16>(a, y_dtype, s);
}

}  // namespace gadei::learner
