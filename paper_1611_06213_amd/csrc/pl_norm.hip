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
// a worker's rows, go to the workspace and are joined in order.
#include <algorithm>

#include "pl_device.h"

namespace gadei::learner {
namespace {

constexpr int kJoinCols = 32, kJoinRows = 8;   // of a workgroup of `join`
constexpr int kSums = 6;
constexpr uint64_t kRowCols = 8 * 1024;        // of a row that 1024 threads hold, eight columns each
constexpr uint64_t kGradCols = 8 * 512;        // backward: 512, for their registers

// Eight columns of a vector of weights, or ones where there is none; past `count`: zeros.
__device__ __forceinline__ void vector8(float (&w)[8], const void *p, int bf16, int64_t at, int count) {
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = 1.0f;
    } else if (bf16) {
        widen8<PS_BF16>(w, count == 8 ? load8<PS_BF16>(p, at) : load8_some<PS_BF16>(p, at, count));
    } else {
        widen8<PS_F32>(w, count == 8 ? load8<PS_F32>(p, at) : load8_some<PS_F32>(p, at, count));
    }
}

template <int DT>
__device__ __forceinline__ void row8(float (&x)[8], const void *p, int64_t at, int count) {
    widen8<DT>(x, count == 8 ? load8<DT>(p, at) : load8_some<DT>(p, at, count));
}

template <int DT>
__device__ __forceinline__ void put8(void *p, int64_t at, const float (&x)[8], int count) {
    if (count == 8) store8<DT>(p, at, x);
    else store_some<DT>(p, at, x, count);
}

__device__ __forceinline__ int count_at(uint64_t cols, uint64_t col) {
    return cols >= col + 8 ? 8 : cols > col ? static_cast<int>(cols - col) : 0;
}

// Sums over the threads of a row: a wave, or a whole workgroup, whose waves' sums go through `lds`
// (two places in turn, so that one barrier is enough).
template <int K>
__device__ __forceinline__ void sum_row(float (&s)[K], float *lds, int *turn) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) s[k] += __shfl_xor(s[k], d);
    const int waves = static_cast<int>(blockDim.x) >> 6;
    if (waves == 1) return;
    float *at = lds + *turn * 16 * kSums;
    *turn ^= 1;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) at[(threadIdx.x >> 6) * K + k] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = 0.0f;
    for (int w = 0; w < waves; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k) s[k] += at[w * K + k];
}

__device__ __forceinline__ float inverse_root(float sum, uint64_t cols, float eps) {
    return 1.0f / sqrtf(sum / static_cast<float>(cols) + eps);
}

// ----------------------------------------------------------------- forward

// What the block leaves in the stream: h of eight columns, from y times ry.
template <int X>
__device__ __forceinline__ void stream8(float (&h)[8], const NormArgs &a, const float (&y)[8], float ry,
                                        uint32_t row, uint64_t col, int count) {
    float x[8], after[8], gate[8];
    row8<X>(x, a.x, row * a.x_ld + static_cast<int64_t>(col), count);
    vector8(after, a.after, a.weight_bf16, static_cast<int64_t>(col), count);
    vector8(gate, a.gate, a.gate_bf16, row / a.per_gate * a.gate_ld + static_cast<int64_t>(col), count);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = a.scale * x[e] + y[e] * ry * after[e] * gate[e];
}

template <int X, int Y, int N, bool BLOCK>
__global__ __launch_bounds__(1024) void norm(NormArgs a) {
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint64_t row64 = static_cast<uint64_t>(block_index()) * blockDim.y + threadIdx.y;
    if (row64 >= a.rows) return;   // a whole wave, of those that no barrier waits for
    const uint32_t row = static_cast<uint32_t>(row64);
    float h[N][8];
    float y[N][8];
    float s[1] = {0.0f};
    if constexpr (BLOCK) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t col = 8 * (threadIdx.x + static_cast<uint64_t>(i) * blockDim.x);
            row8<Y>(y[i], a.y, row * a.y_ld + static_cast<int64_t>(col), count_at(a.cols, col));
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += y[i][e] * y[i][e];
        }
        float ry = 1.0f;
        if (a.after != nullptr) {
            sum_row(s, lds, &turn);
            ry = inverse_root(s[0], a.cols, a.eps);
        }
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t col = 8 * (threadIdx.x + static_cast<uint64_t>(i) * blockDim.x);
            const int count = count_at(a.cols, col);
            stream8<X>(h[i], a, y[i], ry, row, col, count);
            if (count) put8<X>(a.out, row * a.out_ld + static_cast<int64_t>(col), h[i], count);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint64_t col = 8 * (threadIdx.x + static_cast<uint64_t>(i) * blockDim.x);
            row8<X>(h[i], a.x, row * a.x_ld + static_cast<int64_t>(col), count_at(a.cols, col));
        }
    }
    if (a.normed == nullptr) return;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += h[i][e] * h[i][e];
    sum_row(s, lds, &turn);
    const float rh = inverse_root(s[0], a.cols, a.eps);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const uint64_t col = 8 * (threadIdx.x + static_cast<uint64_t>(i) * blockDim.x);
        const int count = count_at(a.cols, col);
        float w[8];
        vector8(w, a.before, a.weight_bf16, static_cast<int64_t>(col), count);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] *= h[i][e] * rh;
        if (count) put8<Y>(a.normed, row * a.normed_ld + static_cast<int64_t>(col), w, count);
    }
}

// Longer rows: a workgroup a row, which it reads again for each sum.
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(1024) void norm_long(NormArgs a) {
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint64_t row64 = block_index();
    if (row64 >= a.rows) return;
    const uint32_t row = static_cast<uint32_t>(row64);
    const uint64_t first = 8 * threadIdx.x, step = 8 * blockDim.x;
    float s[1] = {0.0f}, ry = 1.0f;
    if (BLOCK && a.after != nullptr) {
        for (uint64_t col = first; col < a.cols; col += step) {
            float y[8];
            row8<Y>(y, a.y, row * a.y_ld + static_cast<int64_t>(col), count_at(a.cols, col));
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += y[e] * y[e];
        }
        sum_row(s, lds, &turn);
        ry = inverse_root(s[0], a.cols, a.eps);
        s[0] = 0.0f;
    }
    auto stream = [&](float (&h)[8], uint64_t col, int count) {
        if constexpr (BLOCK) {
            float y[8];
            row8<Y>(y, a.y, row * a.y_ld + static_cast<int64_t>(col), count);
            stream8<X>(h, a, y, ry, row, col, count);
        } else {
            row8<X>(h, a.x, row * a.x_ld + static_cast<int64_t>(col), count);
        }
    };
    for (uint64_t col = first; col < a.cols; col += step) {
        const int count = count_at(a.cols, col);
        float h[8];
        stream(h, col, count);
        if (BLOCK) put8<X>(a.out, row * a.out_ld + static_cast<int64_t>(col), h, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[0] += h[e] * h[e];
    }
    if (a.normed == nullptr) return;
    sum_row(s, lds, &turn);
    const float rh = inverse_root(s[0], a.cols, a.eps);
    for (uint64_t col = first; col < a.cols; col += step) {
        const int count = count_at(a.cols, col);
        float h[8], w[8];
        stream(h, col, count);
        vector8(w, a.before, a.weight_bf16, static_cast<int64_t>(col), count);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] *= h[e] * rh;
        put8<Y>(a.normed, row * a.normed_ld + static_cast<int64_t>(col), w, count);
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

// Eight columns of a row and of the vectors.
template <int X, int Y, bool BLOCK>
struct Eight {
    float h[8], u[8], dz[8], before[8], y[8], dh[8], after[8], gate[8];
    __device__ __forceinline__ void load(const NormGradArgs &a, uint32_t row, uint64_t col, int count) {
        const int64_t c = static_cast<int64_t>(col);
        row8<X>(h, a.h, row * a.h_ld + c, count);
        if (a.dz != nullptr) {
            row8<Y>(dz, a.dz, row * a.dz_ld + c, count);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) dz[e] = 0.0f;
        }
        vector8(before, a.before, a.weight_bf16, c, count);
        if constexpr (BLOCK) {
            row8<Y>(y, a.y, row * a.y_ld + c, count);
            vector8(after, a.after, a.weight_bf16, c, count);
            vector8(gate, a.gate, a.gate_bf16, row / a.per_gate * a.gate_ld + c, count);
        }
        if (a.dh != nullptr) {
            row8<X>(dh, a.dh, row * a.dh_ld + c, count);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) dh[e] = 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) u[e] = dz[e] * before[e];
    }
    // h h, u h; y y, and of p = gate after y: p dh, p u, p h
    __device__ __forceinline__ void sums(float (&s)[kSums]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s[0] += h[e] * h[e];
            s[1] += u[e] * h[e];
            if constexpr (BLOCK) {
                const float p = gate[e] * after[e] * y[e];
                s[2] += y[e] * y[e];
                s[3] += p * dh[e];
                s[4] += p * u[e];
                s[5] += p * h[e];
            }
        }
    }
};

// rh, k1 = rh^2 mean(u h), ry, k2 = ry^2 mean(v y). Without a norm before or after: 0, 0 and 1, 0.
__device__ __forceinline__ f32x4 row_factors(const NormGradArgs &a, const float (&s)[kSums]) {
    const float n = static_cast<float>(a.cols);
    f32x4 r = {0.0f, 0.0f, 1.0f, 0.0f};
    if (a.dz != nullptr) {
        r[0] = inverse_root(s[0], a.cols, a.eps);
        r[1] = r[0] * r[0] * (s[1] / n);
    }
    if (a.after != nullptr) {
        r[2] = inverse_root(s[2], a.cols, a.eps);
        r[3] = r[2] * r[2] * ((s[3] + r[0] * (s[4] - r[1] * s[5])) / n);
    }
    return r;
}

struct Gradients {
    float before[8], after[8], gate[8];   // sums over rows
    __device__ __forceinline__ void zero(float (&x)[8]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0.0f;
    }
};

template <int X, int Y, bool BLOCK>
__device__ __forceinline__ void take_row(const NormGradArgs &a, const Eight<X, Y, BLOCK> &v, f32x4 r,
                                         uint32_t row, uint64_t col, int count, Gradients &sum) {
    float dx[8], dy[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = v.dh[e] + r[0] * (v.u[e] - v.h[e] * r[1]);
        dx[e] = a.scale * d;
        sum.before[e] += v.dz[e] * (v.h[e] * r[0]);
        if constexpr (BLOCK) {
            const float n = v.y[e] * r[2], g = d * v.gate[e];
            sum.gate[e] += d * (n * v.after[e]);
            sum.after[e] += g * n;
            dy[e] = r[2] * (g * v.after[e] - v.y[e] * r[3]);
        }
    }
    if (count == 0) return;
    put8<X>(a.dx, row * a.dx_ld + static_cast<int64_t>(col), dx, count);
    if constexpr (BLOCK) put8<Y>(a.dy, row * a.dy_ld + static_cast<int64_t>(col), dy, count);
}

__device__ __forceinline__ void put_result(const NormGradArgs &a, void *p, int64_t at, float (&x)[8], int count) {
    if (a.accumulate) {
        float old[8];
        vector8(old, p, a.out_bf16, at, count);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] += old[e];
    }
    if (a.out_bf16) put8<PS_BF16>(p, at, x, count);
    else put8<PS_F32>(p, at, x, count);
}

// The gate's sum when its last row, or the worker's, has been taken.
__device__ __forceinline__ void end_gate(const NormGradArgs &a, const Split &sp, uint32_t worker, uint32_t first,
                                         uint32_t row, uint32_t last, uint64_t col, int count, Gradients &sum) {
    if (a.dgate == nullptr) return;
    const uint32_t gate = row / a.per_gate;
    const uint64_t begins = static_cast<uint64_t>(gate) * a.per_gate, ends = begins + a.per_gate;
    if (row + 1 != ends && row + 1 != last) return;
    if (count) {
        if (begins >= first && ends <= last) {
            put_result(a, a.dgate, gate * a.dgate_ld + static_cast<int64_t>(col), sum.gate, count);
        } else {
            const uint64_t slot = 2 * static_cast<uint64_t>(worker) + (begins >= first ? 1 : 0);
            store8<PS_F32>(sp.gate, static_cast<int64_t>(slot * sp.pitch + col), sum.gate);
        }
    }
    sum.zero(sum.gate);
}

__device__ __forceinline__ void end_worker(const NormGradArgs &a, const Split &sp, uint32_t worker, uint64_t col,
                                           int count, const Gradients &sum) {
    if (count == 0) return;
    const int64_t at = static_cast<int64_t>(worker * sp.pitch + col);
    if (a.dbefore != nullptr) store8<PS_F32>(sp.before, at, sum.before);
    if (a.dafter != nullptr) store8<PS_F32>(sp.after, at, sum.after);
}

// A worker is a wave or a workgroup, its rows in registers one after another.
template <int X, int Y, bool BLOCK, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad(NormGradArgs a, Split sp) {
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint32_t worker = block_index() * blockDim.y + threadIdx.y;
    if (worker >= sp.workers) return;   // a whole wave, of those that no barrier waits for
    const uint32_t first = worker * sp.rows, last = min(a.rows - first, sp.rows) + first;
    const uint64_t col = 8 * threadIdx.x;
    const int count = count_at(a.cols, col);
    Gradients sum = {};
    for (uint32_t row = first; row < last; ++row) {
        Eight<X, Y, BLOCK> v;
        v.load(a, row, col, count);
        float s[kSums] = {};
        v.sums(s);
        sum_row(s, lds, &turn);
        take_row(a, v, row_factors(a, s), row, col, count, sum);
        end_gate(a, sp, worker, first, row, last, col, count, sum);
    }
    end_worker(a, sp, worker, col, count, sum);
}

// Longer rows: first their sums, a workgroup a row, ...
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(1024) void row_sums(NormGradArgs a, Split sp) {
    __shared__ float lds[2 * 16 * kSums];
    int turn = 0;
    const uint64_t row = block_index();
    if (row >= a.rows) return;
    float s[kSums] = {};
    for (uint64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * blockDim.x) {
        Eight<X, Y, BLOCK> v;
        v.load(a, static_cast<uint32_t>(row), col, count_at(a.cols, col));
        v.sums(s);
    }
    sum_row(s, lds, &turn);
    if (threadIdx.x == 0) sp.rows_of[row] = row_factors(a, s);
}

// ... then strips of columns.
template <int X, int Y, bool BLOCK>
__global__ __launch_bounds__(256) void norm_grad_long(NormGradArgs a, Split sp, uint32_t strips) {
    const uint64_t worker64 = block_index() / strips;
    if (worker64 >= sp.workers) return;
    const uint32_t worker = static_cast<uint32_t>(worker64);
    const uint32_t first = worker * sp.rows, last = min(a.rows - first, sp.rows) + first;
    const uint64_t col = 8 * (threadIdx.x + 256ull * (block_index() % strips));
    const int count = count_at(a.cols, col);
    Gradients sum = {};
    for (uint32_t row = first; row < last; ++row) {
        Eight<X, Y, BLOCK> v;
        v.load(a, row, col, count);
        take_row(a, v, sp.rows_of[row], row, col, count, sum);
        end_gate(a, sp, worker, first, row, last, col, count, sum);
    }
    end_worker(a, sp, worker, col, count, sum);
}

// The workers' sums, in order: y = 0 and 1 dbefore and dafter, from 2 on the gate that goes from
// worker y - 2 into the next.
__global__ __launch_bounds__(kJoinCols * kJoinRows) void join(NormGradArgs a, Split sp) {
    __shared__ float lds[kJoinRows][kJoinCols];
    const int x = threadIdx.x % kJoinCols, y = threadIdx.x / kJoinCols;
    const uint64_t col = static_cast<uint64_t>(blockIdx.x) * kJoinCols + x;
    void *out = blockIdx.y == 0 ? a.dbefore : blockIdx.y == 1 ? a.dafter : a.dgate;
    if (out == nullptr) return;
    int64_t at = static_cast<int64_t>(col);
    uint32_t from = 0, to = sp.workers;
    const float *p = blockIdx.y == 0 ? sp.before : sp.after;
    uint64_t pitch = sp.pitch;
    float v = 0.0f;
    if (blockIdx.y >= 2) {
        from = blockIdx.y - 2;
        const uint64_t boundary = static_cast<uint64_t>(from + 1) * sp.rows, gate = boundary / a.per_gate;
        const uint64_t begins = gate * a.per_gate, ends = begins + a.per_gate;
        // none crosses here, or it does not begin in this worker's rows
        if (begins == boundary || begins < boundary - sp.rows) return;
        at += static_cast<int64_t>(gate) * a.dgate_ld;
        to = static_cast<uint32_t>((ends - 1) / sp.rows) + 1;
        p = sp.gate;
        pitch = 2 * sp.pitch;
        if (y == 0 && col < a.cols) v = p[(2ull * from + 1) * sp.pitch + col];
        ++from;
    }
    if (col < a.cols) {
#pragma unroll 8
        for (uint32_t w = from + y; w < to; w += kJoinRows) v += p[w * pitch + col];
    }
    lds[y][x] = v;
    __syncthreads();
    if (y != 0 || col >= a.cols) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < kJoinRows; ++i) v += lds[i][x];
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

// Threads of a row of so many columns, eight a thread.
uint32_t threads_of(uint64_t cols) {
    uint32_t t = 64;
    while (t < 1024 && 8ull * t < cols) t *= 2;
    return t;
}

template <int X, int Y, bool BLOCK>
hipError_t launch(const NormArgs &a, hipStream_t s) {
    const uint32_t threads = threads_of(a.cols);
    const uint32_t together = threads == 64 ? 4 : 1;   // rows of a workgroup
    dim3 grid;
    if (!grid_of((a.rows + together - 1ull) / together, threads * together, &grid)) return hipErrorInvalidConfiguration;
    if (a.cols <= kRowCols) norm<X, Y, 1, BLOCK><<<grid, dim3(threads, together), 0, s>>>(a);
    else if (a.cols <= 2 * kRowCols) norm<X, Y, 2, BLOCK><<<grid, threads, 0, s>>>(a);
    else norm_long<X, Y, BLOCK><<<grid, threads, 0, s>>>(a);
    return hipGetLastError();
}

template <int X>
hipError_t launch(const NormArgs &a, int y_dtype, hipStream_t s) {
    if (a.y == nullptr)
        return y_dtype == PS_F32 ? launch<X, PS_F32, false>(a, s) : launch<X, PS_BF16, false>(a, s);
    return y_dtype == PS_F32 ? launch<X, PS_F32, true>(a, s) : launch<X, PS_BF16, true>(a, s);
}

size_t align256(size_t x) { return (x + 255) & ~size_t(255); }

Split split(uint64_t rows, uint64_t cols) {
    Split sp{};
    sp.pitch = (cols + 7) & ~uint64_t(7);
    if (rows == 0) return sp;
    const uint64_t most = cols > kGradCols ? 64 : std::max<uint64_t>(256, 2048 * 64 / threads_of(cols));
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
    } else if (a.cols <= kGradCols) {
        const uint32_t together = threads == 64 ? 4 : 1;
        grid = dim3((sp.workers + together - 1) / together);
        if (threads <= 256) norm_grad<X, Y, BLOCK, 256><<<grid, dim3(threads, together), 0, s>>>(a, sp);
        else norm_grad<X, Y, BLOCK, 512><<<grid, threads, 0, s>>>(a, sp);
    } else {
        if (!grid_of(a.rows, 1024, &grid)) return hipErrorInvalidConfiguration;
        row_sums<X, Y, BLOCK><<<grid, 1024, 0, s>>>(a, sp);
        const uint64_t strips = (a.cols + 2047) / 2048;
        if (!grid_of(strips * sp.workers, 256, &grid)) return hipErrorInvalidConfiguration;
        norm_grad_long<X, Y, BLOCK><<<grid, 256, 0, s>>>(a, sp, static_cast<uint32_t>(strips));
    }
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const bool gates = a.dgate != nullptr && a.rows != 0 && sp.rows % a.per_gate != 0;
    if (a.dbefore == nullptr && a.dafter == nullptr && !gates) return hipSuccess;
    grid = dim3(static_cast<uint32_t>((a.cols + kJoinCols - 1) / kJoinCols), gates ? 1 + sp.workers : 2);
    join<<<grid, kJoinCols * kJoinRows, 0, s>>>(a, sp);
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
           (static_cast<uint64_t>(cols) > kGradCols ? sizeof(f32x4) * static_cast<size_t>(rows) : 0);
}

hipError_t launch_norm_grad(const NormGradArgs &a, int x_dtype, int y_dtype, hipStream_t s) {
    return x_dtype == PS_F32 ? launch<PS_F32>(a, y_dtype, s) : launch<PS_BF16>(a, y_dtype, s);
}

}  // namespace gadei::learner
