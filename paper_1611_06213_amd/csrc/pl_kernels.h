// Internal interface between the host side of a learner's operators (pl_api.cpp) and
// their HIP kernels. Not part of the public C ABI.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

#include "ps_learner.h"

namespace gadei::learner {

constexpr int kCus = 256;   // compute units of an MI355X

// Dropout as the kernels take it: elements whose 16-bit number is below `drop`
// become 0, the others are multiplied by a factor that the caller folds into its own.
// drop == 0: none.
struct Drop {
    uint32_t drop;
    uint32_t k0, k1;   // key
    uint32_t o0, o1;   // offset
};

// rows x cols, each row from x + row * x_ld or, with ids, from
// x + ids[row] * x_ld (zeros where the id is not in 0 .. vocab-1), times `factor`,
// dropped out, to out + row * out_ld.
struct RowsArgs {
    const void *ids;
    const void *x;
    void *out;
    uint64_t vocab;
    int64_t x_ld, out_ld;
    uint32_t rows;
    uint64_t cols;
    float factor;
    Drop drop;
};
enum { kNoIds = -1 };
hipError_t launch_rows(const RowsArgs &a, int id_type, int x_dtype, int out_dtype, hipStream_t s);

// Gradient of an embedding table.
struct GradArgs {
    const void *ids;
    const void *grad;
    void *out;
    int64_t grad_ld, out_ld;
    uint32_t tokens, vocab;
    uint64_t dim;
    float factor;
    int accumulate;
    Drop drop;
    void *workspace;
};
size_t grad_workspace(int64_t tokens, int64_t vocab, int64_t dim);
hipError_t launch_grad(const GradArgs &a, int id_type, int grad_dtype, int out_dtype,
                       hipStream_t s);

struct QuantArgs {
    const void *x;
    int64_t ld;
    int64_t rows, cols;
    uint8_t *values, *values_t;      // either may be null
    uint32_t *scales, *scales_t;
};
hipError_t launch_quantize(const QuantArgs &a, int dtype, bool square, hipStream_t s);
// Two matrices of one type.
hipError_t launch_quantize_two(const QuantArgs &a, const QuantArgs &b, int dtype, bool square, hipStream_t s);

struct MatmulArgs {
    const uint8_t *a, *b;
    const uint32_t *sa, *sb;
    const void *bias;
    void *out;
    int64_t out_ld;
    uint32_t m, n, k;       // k: real columns; rows are padded to whole blocks of 128
    int bias_bf16;
    int relu;
    int accumulate;
    float *partial;         // workspace
    const void *x;          // launch_convert_matmul: what a is made from
    int64_t x_ld;
};
size_t matmul_workspace(int64_t m, int64_t n, int64_t k, int out_dtype);
hipError_t launch_matmul(const MatmulArgs &a, int out_dtype, hipStream_t s);
// Whether two products go in one launch: small ones, whose workgroups all run at once.
bool pairs(const MatmulArgs &a, int a_dtype, const MatmulArgs &b, int b_dtype);
hipError_t launch_matmul_two(const MatmulArgs &a, int a_dtype, const MatmulArgs &b, int b_dtype,
                             hipStream_t s);
// Whether the product of m x k numbers not yet in 8-bit form is one launch, which needs no a, sa or
// workspace.
bool converts(int64_t m, int64_t n, int64_t k);
hipError_t launch_convert_matmul(const MatmulArgs &a, int x_dtype, int out_dtype, hipStream_t s);

// One AdamW step. A plan has an entry for each workgroup, which counts the steps made.
struct AdamwPart {
    void *weight, *grad;   // the part's first elements
    int64_t at;            // where they are in the states, a multiple of 128
    int64_t steps;
    uint32_t count;
    float decay;
};
struct AdamwArgs {
    AdamwPart *plan;
    uint64_t parts;
    void *m, *v;                     // fp32 or 8-bit codes
    uint8_t *m_scales, *v_scales;    // of codes, a byte for each 128
    double log2_beta1, log2_beta2;
    float beta1, beta2, rest1, rest2, eps, lr, factor;   // rest = 1 - beta
    const float *lr_at, *factor_at;  // on the device, or null
    uint64_t seed;
    bool plain;                      // 2^-30 <= eps <= 2^100, rest2 >= 2^-18
};
uint32_t adamw_part();   // elements of a part, at most, a multiple of 128
hipError_t launch_adamw(const AdamwArgs &a, int weight_dtype, int grad_dtype, int bits, bool push, hipStream_t s);

struct MomentsArgs {
    const uint8_t *m, *v, *m_scales, *v_scales;
    void *m_out, *v_out;
    uint64_t room;   // a multiple of 128
};
hipError_t launch_moments(const MomentsArgs &a, int dtype, hipStream_t s);

// The norms after and before a block. Matrices of `rows` x `cols`; vectors may be null.
struct NormArgs {
    const void *x, *y;               // y null: no block
    int64_t x_ld, y_ld;
    uint32_t rows, per_gate;         // rows that share a row of the gate
    uint64_t cols;
    const void *gate, *after, *before;
    int64_t gate_ld;
    int gate_bf16, weight_bf16;
    float scale, eps;
    void *out, *normed;              // either may be null
    int64_t out_ld, normed_ld;
};
hipError_t launch_norm(const NormArgs &a, int x_dtype, int y_dtype, hipStream_t s);

struct NormGradArgs {
    const void *h, *y, *dh, *dz;     // y, dh, dz may be null
    int64_t h_ld, y_ld, dh_ld, dz_ld;
    uint32_t rows, per_gate, gates;
    uint64_t cols;
    const void *gate, *after, *before;
    int64_t gate_ld;
    int gate_bf16, weight_bf16;
    float scale, eps;
    void *dx, *dy;
    int64_t dx_ld, dy_ld;
    void *dgate, *dafter, *dbefore;  // of one type
    int64_t dgate_ld;
    int out_bf16, accumulate;
    void *workspace;
};
size_t norm_grad_workspace(int64_t rows, int64_t cols);
hipError_t launch_norm_grad(const NormGradArgs &a, int x_dtype, int y_dtype, hipStream_t s);

// Products of 8-bit integers with a scale for each row of either factor.
struct Int8QuantArgs {
    const void *x;
    int64_t ld, rows, cols;
    int8_t *values;
    float *scales;
};
hipError_t launch_quantize_int8(const Int8QuantArgs &a, int dtype, hipStream_t s);

struct Int8Args {
    const int8_t *a, *b;
    const float *sa, *sb;
    const void *bias;
    void *out;
    int64_t out_ld;
    uint32_t m, n, k;       // k: real columns; rows are padded to whole blocks of 128
    int bias_bf16;
    int relu;
    int32_t *partial;       // workspace
    const void *x;          // where a is null: what it is made from
    int64_t x_ld;
    int x_bf16;
};
size_t int8_workspace(int64_t m, int64_t n, int64_t k);
// Whether the product of m x k numbers that are not integers yet is one launch, which needs no a, sa
// or workspace.
bool int8_converts(int64_t m, int64_t n, int64_t k);
hipError_t launch_int8(const Int8Args &a, int out_dtype, hipStream_t s);

}  // namespace gadei::learner
