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

/* What is done with a linear layer's sums. */
typedef enum garfield_activation {
  GARFIELD_NO_ACTIVATION = 0,
  GARFIELD_RELU = 1,      /* max(p, 0); a gradient passes where p > 0 and is 0 elsewhere,
                             whatever it was */
  GARFIELD_GELU = 2,      /* p Phi(p), Phi the normal distribution's */
  GARFIELD_GELU_TANH = 3, /* p (1 + tanh(sqrt(2 / pi) (p + 0.044715 p^3))) / 2 */
  GARFIELD_SILU = 4       /* p / (1 + exp(-p)) */
} garfield_activation;

/*
 * A linear layer of 16- or 32-bit matrices with its epilogue: of every token and output
 *   p = sum_k x[t][k] w[j][k] + bias[j],  out[t][j] = act(p) + residual[t][j].
 * x (tokens x inputs), w (outputs x inputs), residual and out (tokens x outputs) are of
 * `type`; bias (outputs values) is of btype: GARFIELD_F32 or `type`. bias, residual and pre
 * may be NULL; pre gets p, rounded to `type`, for the backward pass. Sums are fp32, and out
 * and pre are rounded once. fp32 products are those of fp32 values.
 * At most 2^20 inputs and outputs (GARFIELD_ETOOBIG beyond). The workspace holds
 * matrices whose rows the product cannot read as they are (their address, distance or length
 * no multiple of 16 bytes), once more, and the fp32 sums of a few columns' shares.
 */
size_t garfield_linear_workspace(const void* x, int type, int64_t tokens, int64_t inputs,
                                 int64_t ldx, const void* w, int64_t outputs, int64_t ldw);
garfield_status garfield_linear(const void* x, int type, int64_t tokens, int64_t inputs,
                                int64_t ldx, const void* w, int64_t outputs, int64_t ldw,
                                const void* bias, int btype, int activation, const void* residual,
                                int64_t ld_residual, void* out, int64_t ld_out, void* pre,
                                int64_t ld_pre, void* workspace, size_t workspace_bytes,
                                void* stream);

/*
 * The gradient of a linear layer's input, on through what came before it:
 *   dx[t][k] = act'(pre[t][k]) sum_j dy[t][j] w[j][k] + residual[t][k],
 * with pre what garfield_linear kept of the layer before (tokens x inputs, NULL with
 * GARFIELD_NO_ACTIVATION), and residual a gradient that reaches the same place by another way
 * (NULL: none). All matrices are of `type`; sums are fp32, dx is rounded once.
 */
size_t garfield_linear_backward_workspace(const void* dy, int type, int64_t tokens,
                                          int64_t outputs, int64_t lddy, const void* w,
                                          int64_t inputs, int64_t ldw);
garfield_status garfield_linear_backward(const void* dy, int type, int64_t tokens, int64_t outputs,
                                         int64_t lddy, const void* w, int64_t inputs, int64_t ldw,
                                         int activation, const void* pre, int64_t ld_pre,
                                         const void* residual, int64_t ld_residual, void* dx,
                                         int64_t lddx, void* workspace, size_t workspace_bytes,
                                         void* stream);

/* dp = act'(pre) dy, values of `type` (rows x cols): from the gradient of garfield_linear's out
 * to that of its sums. */
garfield_status garfield_activation_backward(const void* dy, int type, int64_t rows, int64_t cols,
                                             int64_t lddy, int activation, const void* pre,
                                             int64_t ld_pre, void* dp, int64_t lddp, void* stream);

/*
 * garfield_weight_gradient of an input that is no checkpoint: x (tokens x inputs) is of dy's
 * type. At most 2^20 outputs and inputs.
 */
size_t garfield_linear_weight_gradient_workspace(const void* dy, int type, int64_t tokens,
                                                 int64_t outputs, int64_t lddy, const void* x,
                                                 int64_t inputs, int64_t ldx, int n,
                                                 const int64_t* counts);
garfield_status garfield_linear_weight_gradient(const void* dy, int type, int64_t tokens,
                                                int64_t outputs, int64_t lddy, const void* x,
                                                int64_t inputs, int64_t ldx, int n,
                                                const int64_t* counts, float* dw, int64_t ld_dw,
                                                float* dbias, int64_t ld_dbias, void* workspace,
                                                size_t workspace_bytes, void* stream);

/*
 * The residual around a block, with the norms before and after it: of every token
 *   s = scale * x + gate * N_post(h),  y = N(s),
 * where x is the residual stream, h the block's result, and N a norm of rows
 *   N(v)_c = (v_c - mean) * rstd * weight_c + bias_c  (rms: v_c * rstd * weight_c)
 * with mean = sum_c v_c / cols and rstd = (sum_c (v_c - mean)^2 / cols + eps)^(-1/2); with rms
 * the mean is 0 and there are no biases. x, h, s and y (rows x cols) are of `type`; weights,
 * biases and a gate of columns (cols values each) of wtype: GARFIELD_F32 or `type`.
 */
typedef struct garfield_residual_block {
  int type, wtype;
  int64_t rows, cols;
  int rms;
  float eps, scale;
  const void *weight, *bias;           /* of N; weight NULL: no norm after, no y */
  const void *post_weight, *post_bias; /* of N_post; post_weight NULL: N_post(h) = h */
  const void* gate;                    /* NULL: 1 */
  int64_t ld_gate; /* 0: gate is one value a column; else a matrix of `type` like h */
} garfield_residual_block;

/*
 * s, y and each row's statistics (rows fp32 values; the means are not written with rms and
 * may be NULL then, those of a norm that is not there too). y and y8 (the checkpoint of y's
 * values in 32 bits) may be NULL. s is rounded once; y is formed from s in 32 bits, before
 * it is rounded. The means' sums are kept as garfield_layernorm keeps them.
 */
garfield_status garfield_residual_norm(const garfield_residual_block* b, const void* x,
                                       int64_t ldx, const void* h, int64_t ldh, void* s,
                                       int64_t lds, void* y, int64_t ldy, float* mean, float* rstd,
                                       float* post_mean, float* post_rstd,
                                       const garfield_block8* y8, void* stream);

/* The gradients of each worker: worker w's row at weight + w * ld_weight, and so on (cols
 * fp32 values each). NULL where one is not asked for, or has no parameter. */
typedef struct garfield_residual_gradients {
  float *weight, *bias, *post_weight, *post_bias, *gate;
  int64_t ld_weight, ld_bias, ld_post_weight, ld_post_bias, ld_gate;
} garfield_residual_gradients;

/*
 * Its backward pass, from the gradients of s by other ways (ds) and of y (dy): NULL where
 * there is none, dy also where b->weight is NULL. With g the whole gradient of s,
 *   g = ds + N'(dy),  dx = scale * g,  dh = N_post'(gate * g),
 *   dgate = g * N_post(h)  (by tokens: dgate, a matrix of `type`; by columns: in `gradients`),
 * and the weights' and biases' gradients as garfield_layernorm_backward's. s (needed where dy
 * is given), h and the statistics are the forward pass's. dx, dh and dgate may be NULL.
 */
size_t garfield_residual_norm_backward_workspace(const garfield_residual_block* b, int n,
                                                 const int64_t* counts);
garfield_status garfield_residual_norm_backward(
    const garfield_residual_block* b, const void* ds, int64_t ldds, const void* dy, int64_t lddy,
    const void* s, int64_t lds, const void* h, int64_t ldh, const float* mean, const float* rstd,
    const float* post_mean, const float* post_rstd, void* dx, int64_t lddx, void* dh,
    int64_t lddh, void* dgate, int64_t lddgate, int n, const int64_t* counts,
    const garfield_residual_gradients* gradients, void* workspace, size_t workspace_bytes,
    void* stream);

/* A tensor of every worker's gradient: worker w's `length` values of `type`, next to each
 * other, at values + w * ld elements. */
typedef struct garfield_gradient {
  void* values;
  int64_t length, ld;
  int type;
} garfield_gradient;

/*
 * Each worker's gradient norm over `count` tensors (a HOST array, read before the call
 * returns), norms[w] = (sum of all its values' squares)^(1/2), and its gradient clipped:
 *   out = value * (norm > max_norm ? max_norm / norm : 1),
 * the tensors one after the other into worker w's row of fp32 values at out + w * ld_out, or
 * in place with out NULL (values are then rounded once to their type). What is written must
 * share no memory with another tensor, or with any with out (GARFIELD_EINVAL). Squares are added
 * up in 64 bits. A worker with an infinite value gets zeros and, for the infinities, NaN (with
 * max_norm infinite its values as they are); one with a NaN gets NaN throughout: norms says which.
 * At most 2^20 tensors, each of at most 2^34 values a worker (GARFIELD_ETOOBIG).
 */
size_t garfield_clip_workspace(const garfield_gradient* tensors, int count, int n);
garfield_status garfield_gradient_norms(const garfield_gradient* tensors, int count, int n,
                                        float* norms, void* workspace, size_t workspace_bytes,
                                        void* stream);
garfield_status garfield_clip_gradients(const garfield_gradient* tensors, int count, int n,
                                        float max_norm, float* norms, float* out, int64_t ld_out,
                                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif
