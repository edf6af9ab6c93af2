/*
 * garfield_worker.h -- a worker's operators: what comes before the aggregation
 * rules of garfield.h. The n workers' tokens lie one worker after the other in
 * a T x D matrix, and each worker's own weight gradient is written to its row
 * of the n x d fp32 matrix the rules take.
 *
 * Conventions, beyond those of garfield.h:
 *   - Pointers named x, y, dy, dx, out, weight, bias, mean, rstd, dweight,
 *     dbias, dw and workspace are DEVICE pointers owned by the caller, aligned
 *     to their element. A matrix has its columns next to each other and its
 *     rows `ld` elements apart (ld >= columns); any ld and any alignment of
 *     the element's own size is taken. Outputs must not overlap inputs.
 *   - counts is a HOST array of n values, the tokens of each worker (0 is
 *     allowed); it is read before the call returns. n <= GARFIELD_NMAX.
 *   - Nothing is kept between calls and no scratch is shared: what a call
 *     needs is the caller's `workspace` (256-byte aligned, at least as many
 *     bytes as the function's _workspace names, NULL if that is 0). Calls on
 *     several streams may overlap when their workspaces differ. A call
 *     enqueues kernels only, so it can be captured in a graph.
 *   - Sizes of zero are allowed (sums over nothing are 0), except the columns
 *     of a layer norm.
 *   - A matrix has at most 2^25 rows, 2^30 columns and 2^34 values (its columns
 *     rounded up to 512); GARFIELD_ETOOBIG beyond.
 *   - Infinities and NaN are allowed and stay where they come from: a row of
 *     a layer norm, a token of a product, a worker's gradient. Another row,
 *     token or worker never sees them.
 *   - Results do not depend on the launch's timing: the same call gives the
 *     same bits.
 */
#ifndef GARFIELD_WORKER_H
#define GARFIELD_WORKER_H

#include <stddef.h>
#include <stdint.h>

#include "garfield.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum garfield_type {
  GARFIELD_F32 = 0,
  GARFIELD_BF16 = 1,
  GARFIELD_F16 = 2
} garfield_type;

/* Values that share one exponent. */
#define GARFIELD_BLOCK 128

/*
 * A rows x cols matrix in 8-bit blocks. Row r's values are e4m3 codes (4
 * exponent bits, 3 mantissa bits, no infinity) at values[r * ld_values + c];
 * its block b (columns 128 b to 128 b + 127) has the exponent
 * s = exponents[r * ld_exponents + b] - 127, and value c stands for
 * code * 2^s. s is the smallest integer, at least -117, with
 * max |finite value of the block| <= 448 * 2^s, so no value is clipped; codes
 * are rounded to nearest, ties to even (and stop at 240 where s = 120: 256 * 2^120
 * is beyond fp32); infinities and NaN become NaN.
 * Every such value is exact in bf16.
 * Rows are padded: codes 0 up to a multiple of 128 columns, exponents 127 up
 * to a multiple of four blocks. values is 16-byte aligned with ld_values a
 * multiple of 16 and at least the padded columns; exponents is 4-byte aligned
 * with ld_exponents a multiple of 4 and at least the padded blocks. Functions
 * that read blocks read the padding too; those that write them write it.
 */
typedef struct garfield_block8 {
  uint8_t* values;
  uint8_t* exponents;
  int64_t rows, cols, ld_values, ld_exponents;
} garfield_block8;

/*
 * An 8-bit checkpoint of x (rows x cols, of `type`): out holds x itself, or its
 * transpose if `transposed` (out is then cols x rows, blocks along x's rows).
 */
garfield_status garfield_checkpoint(const void* x, int type, int64_t rows, int64_t cols,
                                    int64_t ld, int transposed, const garfield_block8* out,
                                    void* stream);

/* The values of a checkpoint, rounded once to `type`. */
garfield_status garfield_restore(const garfield_block8* c, void* out, int type, int64_t ld,
                                 void* stream);

/*
 * Layer norm of each row of x (rows x cols, of `type`):
 *   mean = sum_c x_c / cols,  rstd = (sum_c (x_c - mean)^2 / cols + eps)^(-1/2),
 *   y_c = (x_c - mean) * rstd * weight_c + bias_c.
 * weight and bias (cols values of wtype: GARFIELD_F32 or `type`; bias may be
 * NULL). mean, rstd: rows fp32 values each. y (of `type`), y8 and x8 may be
 * NULL each: y8 is the checkpoint of y's values in 32 bits (before they are
 * rounded to `type`), x8 that of x. Statistics and y are formed in fp32, the
 * variance from the differences to the mean; the mean's sum is kept in fp64 but
 * for differences within a row, so a row of equal values has exactly that mean.
 */
garfield_status garfield_layernorm(const void* x, int type, int64_t rows, int64_t cols,
                                   int64_t ldx, const void* weight, const void* bias, int wtype,
                                   float eps, void* y, int64_t ldy, float* mean, float* rstd,
                                   const garfield_block8* y8, const garfield_block8* x8,
                                   void* stream);

/*
 * Its backward pass, with the weight's gradient of each worker. With
 * h_c = (x_c - mean) * rstd and g_c = dy_c * weight_c, a row's
 *   dx_c = rstd * (g_c - sum_j g_j / cols - h_c * sum_j g_j h_j / cols),
 * and over the tokens of worker w (sum of counts = rows)
 *   dweight[w][c] = sum dy_c h_c,  dbias[w][c] = sum dy_c.
 * dy and dx are of `type`. x is given as a matrix of `type` or, with x NULL,
 * as a checkpoint x8. mean and rstd are the forward pass's. dx, dweight and
 * dbias may be NULL each; worker w's row starts at dweight + w * ld_dweight
 * (dbias likewise). A worker of no tokens gets zeros.
 */
size_t garfield_layernorm_backward_workspace(int64_t rows, int64_t cols, int n,
                                             const int64_t* counts);
garfield_status garfield_layernorm_backward(
    const void* dy, int type, int64_t rows, int64_t cols, int64_t lddy, const void* x, int64_t ldx,
    const garfield_block8* x8, const float* mean, const float* rstd, const void* weight, int wtype,
    void* dx, int64_t lddx, int n, const int64_t* counts, float* dweight, int64_t ld_dweight,
    float* dbias, int64_t ld_dbias, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The product of 8-bit blocks: out[m][j] = sum_k x[m][k] w[j][k] + bias[j],
 * x->rows x w->rows values of `type` (x->cols == w->cols). bias: fp32, may be
 * NULL. Products are exact, sums are fp32, out is rounded once. With `fast` the
 * product may run on the scaled 8-bit matrix instruction, at up to twice the
 * rate: of every eight products that it adds at a time it drops what is below
 * 2^-13 of the largest one's binade. That is at most 2^-10 of the products'
 * magnitudes added up; measured, 1.5e-5 (normal values) to 4.3e-5 (activations
 * with a few far larger channels) of the result, root mean square.
 * Up to 32 tokens, and up to 64 that are not cut into shares, it changes nothing.
 * The workspace is 0, or holds the fp32 sums of a few columns' shares: at most
 * 3 tiles of 64 x 64 for each of the card's compute units (13 MB on 256).
 */
size_t garfield_linear8_workspace(int64_t tokens, int64_t outputs, int64_t inputs);
garfield_status garfield_linear8(const garfield_block8* x, const garfield_block8* w,
                                 const float* bias, int fast, void* out, int type, int64_t ld,
                                 void* workspace, size_t workspace_bytes, void* stream);

/*
 * The weight gradient of a linear layer for each worker, from the gradient of
 * its output (tokens x outputs, of `type`) and the checkpoint of its input
 * (x->rows = tokens = sum of counts): over the tokens t of worker w
 *   dw[w][j][k] = sum_t dy[t][j] x[t][k]  (outputs x x->cols fp32, contiguous,
 *                                          worker w's at dw + w * ld_dw),
 *   dbias[w][j] = sum_t dy[t][j]          (dbias may be NULL).
 * Every product is exact (dy of more bits than bf16 is split into bf16 parts,
 * two of fp16 and three of fp32: fp32 values below about 2^-110 may lose their
 * last parts), sums are fp32. At most 2^24 outputs, rows of x at most 2^26 bytes
 * apart (GARFIELD_ETOOBIG beyond). The workspace holds dy's parts, two bytes a
 * value each with the outputs rounded up to eight (bf16 too where dy, its rows or
 * the outputs are no multiple of 16 bytes or eight values), and where tokens are
 * cut into up to 16 shares the gradients of each share.
 */
size_t garfield_weight_gradient_workspace(const void* dy, int type, int64_t tokens,
                                          int64_t outputs, int64_t inputs, int64_t lddy, int n,
                                          const int64_t* counts);
garfield_status garfield_weight_gradient(const void* dy, int type, int64_t tokens,
                                         int64_t outputs, int64_t lddy, const garfield_block8* x,
                                         int n, const int64_t* counts, float* dw, int64_t ld_dw,
                                         float* dbias, int64_t ld_dbias, void* workspace,
                                         size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif
