/*
 * ps_learner.h -- C ABI of a learner's operators on one gfx950 GPU: what a
 * learner computes between a pull and a push with the layers that hold most of
 * the server's parameters (ps.h): embedding tables and fully connected layers,
 * and the dropout between them.
 *
 *   - A learner pulls a replica, reads its layers' weights where they lie in it
 *     (any element boundary), and writes their gradients where they belong in its
 *     gradient row, which it then pushes (Sec. 2.1, 4.1 of arXiv 1611.06213).
 *   - Every call enqueues its kernels on `stream` (a hipStream_t; NULL = the null
 *     stream) and returns without waiting. It allocates nothing: where scratch
 *     memory is needed, the caller passes `workspace` of at least the bytes that
 *     the matching *_workspace call names, free again once the work has completed.
 *     All calls can be captured in a HIP graph. Calls hold no state, so any thread
 *     may make them.
 *   - Matrices are row-major with unit column stride and a row stride `ld` in
 *     elements of at least their columns (any value for a single row). Pointers are
 *     device pointers on the device that is current, aligned to their elements;
 *     16-byte alignment of bases and rows is not needed. No output may overlap an
 *     input or another output, except that pl_dropout may work in place (out == x
 *     with equal strides).
 *   - Element types are PS_F32 and PS_BF16. Sums are held in fp32 and rounded once
 *     to the output's type (nearest even); an 8-bit product with a bf16 result loses more
 *     (see pl_matmul_fp8). Results do not depend on scheduling: equal calls give equal
 *     bits.
 *
 * Status codes and their names are ps.h's: PS_OK, PS_EINVAL (a refused argument;
 * nothing was enqueued), PS_ENOMEM (workspace too small; nothing was enqueued),
 * PS_EHIP (a launch failed). pl_last_error() describes the last failure on this
 * thread.
 */
#ifndef GADEI_PS_LEARNER_H
#define GADEI_PS_LEARNER_H

#include <stddef.h>
#include <stdint.h>

#include "ps.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Types of token ids. */
enum { PL_I32 = 0, PL_I64 = 1 };

/* Dropout by numbers computed from their position, so that no mask is stored:
 * the backward pass names the same seed and offset and computes it again.
 *
 * Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as
 * 1, 2, 3; 2011) with the counter (column >> 3, row, offset low, offset high) and the
 * key (seed low, seed high) gives four 32-bit words: 16-bit numbers for the columns
 * 8j .. 8j+7 of a row, the low half of a word before the high one. With
 * d = floor(65536 p + 0.5), an element is kept if its number is at least d, and
 * multiplied by 65536 / (65536 - d): p counts to the nearest 2^-16, and the
 * expectation is exact for the p that is used. p = 1 drops everything; a dropped
 * element is 0 whatever it was (NaN too). */
typedef struct pl_drop {
    float p;          /* 0 .. 1 */
    uint64_t seed;
    uint64_t offset;  /* another one for each call that is to drop others */
} pl_drop;

/* out[t, c] = scale * table[ids[t], c], then dropout (drop may be NULL) with t as the
 * row. An id outside 0 .. vocab-1 is no token (padding): its row is zeros. tokens,
 * vocab and dim may be 0; tokens < 2^32, dim <= 2^32. */
int pl_embedding(const void *ids, int id_type, int64_t tokens, const void *table, int table_dtype,
                 int64_t vocab, int64_t dim, int64_t table_ld, float scale, const pl_drop *drop,
                 void *out, int out_dtype, int64_t out_ld, void *stream);

/* The gradient of pl_embedding for its table, from grad, that of its result:
 *   out[v, c] = scale * sum over t with ids[t] == v of drop(grad)[t, c]
 * for every row v (zeros for ids that do not occur), with accumulate added to what
 * out holds instead (rows whose id does not occur are then not touched). The tokens
 * are sorted by id first; a row's terms are then added in an order that depends on
 * the ids and the sizes alone. tokens < 2^31, vocab <= 2^31. */
int pl_embedding_grad(const void *ids, int id_type, int64_t tokens, const void *grad,
                      int grad_dtype, int64_t grad_ld, int64_t dim, float scale,
                      const pl_drop *drop, void *out, int out_dtype, int64_t out_ld,
                      int64_t vocab, int accumulate, void *workspace, size_t workspace_bytes,
                      void *stream);
size_t pl_embedding_grad_workspace(int64_t tokens, int64_t vocab, int64_t dim);

/* out = drop(x) for a matrix of rows x cols (a vector: one row); of a gradient, the
 * backward pass of the same call. rows < 2^32, cols <= 2^32. */
int pl_dropout(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld,
               const pl_drop *drop, void *out, int64_t out_ld, void *stream);

/* A matrix in 8-bit floating point (OCP e4m3: 4 exponent and 3 mantissa bits, largest
 * value 448) with a scale for each block of 128 columns of a row:
 *   element (r, c) = values[r * pl_fp8_ld(cols) + c] * 2^(s - 127),
 *   s = byte c / 128 % 4 of word scales[(c / 512) * rows + r].
 * The values' rows are padded with zeros to whole blocks. Both arrays lie on 16-byte
 * boundaries. A scale is a power of two because the matrix instructions take such
 * scales with their operands; the elements lose nothing by it but one of e4m3's 17
 * binades at most. */
typedef struct pl_fp8 {
    void *values;      /* pl_fp8_values_bytes(rows, cols) bytes */
    uint32_t *scales;  /* pl_fp8_scales_bytes(rows, cols) bytes */
} pl_fp8;
int64_t pl_fp8_ld(int64_t cols);
size_t pl_fp8_values_bytes(int64_t rows, int64_t cols);
size_t pl_fp8_scales_bytes(int64_t rows, int64_t cols);

/* x (rows x cols) to 8 bits: `out` in its own layout (blocks along x's rows) and/or
 * `out_t` transposed, as a cols x rows matrix (blocks along x's columns). One of them may
 * be NULL; x is read once for both. square: one scale for each 128 x 128 tile of x instead
 * (for weights: both layouts then hold the same values). A block's scale is the least
 * 2^e, e >= -126, with max|x| <= 448 * 2^e over its finite elements; elements are rounded
 * to nearest even. NaN and infinities become NaN. rows, cols < 2^31. */
int pl_quantize_fp8(const void *x, int dtype, int64_t rows, int64_t cols, int64_t ld, int square,
                    const pl_fp8 *out, const pl_fp8 *out_t, void *stream);

/* out = a b^T (+ bias) (then max(., 0) with relu; a NaN stays) for a (m x k) and b (n x k),
 * out m x n; with accumulate added to what out holds. bias: n values or NULL. relu and
 * bias with accumulate are refused. m, n, k may be 0 (k = 0: a sum of no terms);
 * m, n <= 2^28, k <= 2^22.
 *
 * An fp32 result carries fp32 sums of the products of the elements, which count as they are but
 * in blocks whose scale is below 2^-124, where they are rounded to multiples of 2^-133.
 *
 * For a bf16 result the 8-bit matrix instructions are used, at twice the rate: of eight neighbouring
 * products they keep 13 bits below the largest, and they add the eights' sums in fp32. That is an
 * error of about 2^-19 of the sum of the products' magnitudes (root mean square), which bf16's
 * rounding covers unless large products cancel. Where they may, take an fp32 result. */
int pl_matmul_fp8(int64_t m, int64_t n, int64_t k, const pl_fp8 *a, const pl_fp8 *b,
                  const void *bias, int bias_dtype, int relu, void *out, int out_dtype,
                  int64_t out_ld, int accumulate, void *workspace, size_t workspace_bytes,
                  void *stream);
size_t pl_matmul_fp8_workspace(int64_t m, int64_t n, int64_t k, int out_dtype);

/* A fully connected layer: pl_quantize_fp8 of x (m x k, blocks along its rows), then
 * pl_matmul_fp8 with the weights w (n x k) -- the same result, in fewer launches where
 * x is small. */
int pl_linear_fp8(const void *x, int dtype, int64_t m, int64_t k, int64_t ld, int64_t n,
                  const pl_fp8 *w, const void *bias, int bias_dtype, int relu, void *out,
                  int out_dtype, int64_t out_ld, void *workspace, size_t workspace_bytes,
                  void *stream);
size_t pl_linear_fp8_workspace(int64_t m, int64_t n, int64_t k, int dtype, int out_dtype);

/* The gradients of x w^T (x m x k, w n x k) from grad (m x n), that of the result: out
 * (m x k) = grad w, from w transposed in 8 bits (w_t, k x n), and weight_out (n x k) = grad^T x,
 * with accumulate added to what it holds. grad is quantised along its rows for the first
 * product, grad and x along their columns for the second. m, n <= 2^22, k <= 2^28. Each result's
 * sums are as pl_matmul_fp8 has them for its type. */
int pl_linear_fp8_grad(const void *x, int x_dtype, int64_t x_ld, const void *grad, int grad_dtype,
                       int64_t grad_ld, int64_t m, int64_t n, int64_t k, const pl_fp8 *w_t, void *out,
                       int out_dtype, int64_t out_ld, void *weight_out, int weight_dtype,
                       int64_t weight_ld, int accumulate, void *workspace, size_t workspace_bytes,
                       void *stream);
size_t pl_linear_fp8_grad_workspace(int64_t m, int64_t n, int64_t k, int out_dtype, int weight_dtype);

/* Message for the last failed call on this thread ("" if none). */
const char *pl_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* GADEI_PS_LEARNER_H */
