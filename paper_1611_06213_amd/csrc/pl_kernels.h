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

}  // namespace gadei::learner
