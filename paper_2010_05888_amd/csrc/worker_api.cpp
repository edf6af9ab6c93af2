// C-ABI of the worker's operators: argument validation and dispatch. See
// include/garfield_worker.h.

#include <hip/hip_runtime.h>

#include "garfield_worker.h"
#include "internal.h"
#include "worker.h"

namespace garfield {
namespace {

// Beyond these a launch would have more than 2^32 threads, or an index into a
// row would not fit. Offsets into a matrix are 64-bit.
constexpr int64_t kMaxRows = int64_t{1} << 25;
constexpr int64_t kMaxCols = int64_t{1} << 30;
constexpr int64_t kMaxBlocks = int64_t{1} << 27;  // of one matrix, padded
// Weight gradients address 32 tokens with 32 bits.
constexpr int64_t kMaxOutputs = int64_t{1} << 24;
constexpr int64_t kMaxStride = int64_t{1} << 26;

garfield_status status_of(hipError_t e) {
  if (e == hipSuccess) return GARFIELD_OK;
  (void)hipGetLastError();
  return GARFIELD_EHIP;
}

int64_t element_bytes(int type) { return type == GARFIELD_F32 ? 4 : 2; }
bool is_type(int type) { return type >= GARFIELD_F32 && type <= GARFIELD_F16; }

bool aligned(const void* p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

garfield_status check_size(int64_t rows, int64_t cols) {
  if (rows < 0 || cols < 0) return GARFIELD_EINVAL;
  if (rows > kMaxRows || cols > kMaxCols) return GARFIELD_ETOOBIG;
  if (rows * ((cols + 511) / 512 * 4) > kMaxBlocks) return GARFIELD_ETOOBIG;
  return GARFIELD_OK;
}

// A matrix that the call reads or writes.
bool matrix_ok(const void* p, int type, int64_t rows, int64_t cols, int64_t ld) {
  if (rows == 0 || cols == 0) return true;
  return p && aligned(p, element_bytes(type)) && ld >= cols;
}

bool vector_ok(const void* p, int64_t bytes, int64_t length) {
  return length == 0 || (p && aligned(p, bytes));
}

bool block8_ok(const garfield_block8* b, int64_t rows, int64_t cols) {
  if (!b || b->rows != rows || b->cols != cols) return false;
  if (rows == 0 || cols == 0) return true;
  const int64_t blocks = (cols + GARFIELD_BLOCK - 1) / GARFIELD_BLOCK;
  return b->values && aligned(b->values, 16) && b->ld_values % 16 == 0 &&
         b->ld_values >= blocks * GARFIELD_BLOCK && b->exponents && aligned(b->exponents, 4) &&
         b->ld_exponents % 4 == 0 && b->ld_exponents >= (blocks + 3) / 4 * 4;
}

garfield_status check_counts(int n, const int64_t* counts, int64_t rows) {
  if (n < 1 || !counts) return GARFIELD_EINVAL;
  if (n > GARFIELD_NMAX) return GARFIELD_ETOOBIG;
  int64_t left = rows;
  for (int w = 0; w < n; ++w) {
    if (counts[w] < 0 || counts[w] > left) return GARFIELD_EINVAL;
    left -= counts[w];
  }
  return left == 0 ? GARFIELD_OK : GARFIELD_EINVAL;
}

// A worker's gradients: n rows of `length` values, `ld` apart.
bool gradient_ok(const float* p, int n, int64_t length, int64_t ld) {
  return !p || length == 0 || (aligned(p, 4) && (n == 1 || ld >= length));
}

bool workspace_ok(const void* p, size_t bytes, size_t need) {
  return need == 0 || (p && aligned(p, 256) && bytes >= need);
}

}  // namespace
}  // namespace garfield

using namespace garfield;

extern "C" {

garfield_status garfield_checkpoint(const void* x, int type, int64_t rows, int64_t cols,
                                    int64_t ld, int transposed, const garfield_block8* out,
                                    void* stream) {
  if (!is_type(type)) return GARFIELD_EINVAL;
  const int64_t to_rows = transposed ? cols : rows, to_cols = transposed ? rows : cols;
  garfield_status st = check_size(rows, cols);
  if (st == GARFIELD_OK) st = check_size(to_rows, to_cols);
  if (st != GARFIELD_OK) return st;
  if (!matrix_ok(x, type, rows, cols, ld) || !block8_ok(out, to_rows, to_cols))
    return GARFIELD_EINVAL;
  if (rows == 0 || cols == 0) return GARFIELD_OK;
  return status_of(enqueue_checkpoint(x, type, rows, cols, ld, transposed != 0, *out,
                                      static_cast<hipStream_t>(stream)));
}

garfield_status garfield_restore(const garfield_block8* c, void* out, int type, int64_t ld,
                                 void* stream) {
  if (!c || !is_type(type)) return GARFIELD_EINVAL;
  const garfield_status st = check_size(c->rows, c->cols);
  if (st != GARFIELD_OK) return st;
  if (!block8_ok(c, c->rows, c->cols) || !matrix_ok(out, type, c->rows, c->cols, ld))
    return GARFIELD_EINVAL;
  if (c->rows == 0 || c->cols == 0) return GARFIELD_OK;
  return status_of(enqueue_restore(*c, out, type, ld, static_cast<hipStream_t>(stream)));
}

garfield_status garfield_layernorm(const void* x, int type, int64_t rows, int64_t cols,
                                   int64_t ldx, const void* weight, const void* bias, int wtype,
                                   float eps, void* y, int64_t ldy, float* mean, float* rstd,
                                   const garfield_block8* y8, const garfield_block8* x8,
                                   void* stream) {
  if (!is_type(type) || (wtype != GARFIELD_F32 && wtype != type)) return GARFIELD_EINVAL;
  if (!(eps >= 0.0f)) return GARFIELD_EINVAL;
  const garfield_status st = check_size(rows, cols);
  if (st != GARFIELD_OK) return st;
  if (cols == 0) return GARFIELD_EINVAL;
  if (!matrix_ok(x, type, rows, cols, ldx) || (y && !matrix_ok(y, type, rows, cols, ldy)) ||
      !vector_ok(weight, element_bytes(wtype), cols) ||
      (bias && !vector_ok(bias, element_bytes(wtype), cols)) || !vector_ok(mean, 4, rows) ||
      !vector_ok(rstd, 4, rows) || (y8 && !block8_ok(y8, rows, cols)) ||
      (x8 && !block8_ok(x8, rows, cols)))
    return GARFIELD_EINVAL;
  if (rows == 0) return GARFIELD_OK;
  LayerNorm a = {};
  a.rows = rows;
  a.cols = cols;
  a.x = x;
  a.weight = weight;
  a.bias = bias;
  a.ldx = ldx;
  a.weight_f32 = wtype == GARFIELD_F32;
  a.eps = eps;
  a.share = 1.0 / static_cast<double>(cols);
  a.y = y;
  a.ldy = ldy;
  a.mean = mean;
  a.rstd = rstd;
  if (y8) a.y8 = *y8;
  if (x8) a.x8 = *x8;
  return status_of(enqueue_layernorm(a, type, static_cast<hipStream_t>(stream)));
}

size_t garfield_layernorm_backward_workspace(int64_t rows, int64_t cols, int n,
                                             const int64_t* counts) {
  if (check_size(rows, cols) != GARFIELD_OK || check_counts(n, counts, rows) != GARFIELD_OK)
    return 0;
  return layernorm_backward_bytes(layernorm_backward_chunks(rows, cols, n, counts), cols);
}

garfield_status garfield_layernorm_backward(
    const void* dy, int type, int64_t rows, int64_t cols, int64_t lddy, const void* x, int64_t ldx,
    const garfield_block8* x8, const float* mean, const float* rstd, const void* weight, int wtype,
    void* dx, int64_t lddx, int n, const int64_t* counts, float* dweight, int64_t ld_dweight,
    float* dbias, int64_t ld_dbias, void* workspace, size_t workspace_bytes, void* stream) {
  if (!is_type(type) || (wtype != GARFIELD_F32 && wtype != type)) return GARFIELD_EINVAL;
  garfield_status st = check_size(rows, cols);
  if (st == GARFIELD_OK) st = check_counts(n, counts, rows);
  if (st != GARFIELD_OK) return st;
  if (cols == 0) return GARFIELD_EINVAL;
  if (!matrix_ok(dy, type, rows, cols, lddy) || (dx && !matrix_ok(dx, type, rows, cols, lddx)) ||
      (x ? !matrix_ok(x, type, rows, cols, ldx) : rows > 0 && !block8_ok(x8, rows, cols)) ||
      !vector_ok(weight, element_bytes(wtype), cols) || !vector_ok(mean, 4, rows) ||
      !vector_ok(rstd, 4, rows) || !gradient_ok(dweight, n, cols, ld_dweight) ||
      !gradient_ok(dbias, n, cols, ld_dbias))
    return GARFIELD_EINVAL;
  if (!dx && !dweight && !dbias) return GARFIELD_OK;
  const Chunks chunks = layernorm_backward_chunks(rows, cols, n, counts);
  if (!workspace_ok(workspace, workspace_bytes, layernorm_backward_bytes(chunks, cols)))
    return GARFIELD_EINVAL;
  LayerNormBackward a = {};
  a.rows = rows;
  a.cols = cols;
  a.dy = dy;
  a.x = x;
  a.weight = weight;
  a.lddy = lddy;
  a.ldx = ldx;
  if (!x && x8) a.x8 = *x8;
  a.weight_f32 = wtype == GARFIELD_F32;
  a.mean = mean;
  a.rstd = rstd;
  a.dx = dx;
  a.lddx = lddx;
  a.dweight = dweight;
  a.dbias = dbias;
  a.ld_dweight = ld_dweight;
  a.ld_dbias = ld_dbias;
  return status_of(
      enqueue_layernorm_backward(a, type, chunks, workspace, static_cast<hipStream_t>(stream)));
}

size_t garfield_linear8_workspace(int64_t tokens, int64_t outputs, int64_t inputs) {
  if (check_size(tokens, inputs) != GARFIELD_OK || check_size(outputs, inputs) != GARFIELD_OK)
    return 0;
  return linear8_bytes(tokens, outputs, inputs);
}

garfield_status garfield_linear8(const garfield_block8* x, const garfield_block8* w,
                                 const float* bias, int fast, void* out, int type, int64_t ld,
                                 void* workspace, size_t workspace_bytes, void* stream) {
  if (!x || !w || !is_type(type) || x->cols != w->cols) return GARFIELD_EINVAL;
  garfield_status st = check_size(x->rows, x->cols);
  if (st == GARFIELD_OK) st = check_size(w->rows, w->cols);
  if (st == GARFIELD_OK) st = check_size(x->rows, w->rows);
  if (st != GARFIELD_OK) return st;
  if (!block8_ok(x, x->rows, x->cols) || !block8_ok(w, w->rows, w->cols) ||
      !matrix_ok(out, type, x->rows, w->rows, ld) || (bias && !aligned(bias, 4)))
    return GARFIELD_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes, linear8_bytes(x->rows, w->rows, x->cols)))
    return GARFIELD_EINVAL;
  if (x->rows == 0 || w->rows == 0) return GARFIELD_OK;
  return status_of(
      enqueue_linear8(*x, *w, bias, fast != 0, out, type, ld, workspace,
                                   static_cast<hipStream_t>(stream)));
}

size_t garfield_weight_gradient_workspace(const void* dy, int type, int64_t tokens,
                                          int64_t outputs, int64_t inputs, int64_t lddy, int n,
                                          const int64_t* counts) {
  if (!is_type(type) || check_size(tokens, inputs) != GARFIELD_OK ||
      check_size(tokens, outputs) != GARFIELD_OK || check_size(outputs, inputs) != GARFIELD_OK ||
      check_counts(n, counts, tokens) != GARFIELD_OK)
    return 0;
  return weight_gradient_bytes(type, tokens, outputs, inputs, dy, lddy, n, counts);
}

garfield_status garfield_weight_gradient(const void* dy, int type, int64_t tokens,
                                         int64_t outputs, int64_t lddy, const garfield_block8* x,
                                         int n, const int64_t* counts, float* dw, int64_t ld_dw,
                                         float* dbias, int64_t ld_dbias, void* workspace,
                                         size_t workspace_bytes, void* stream) {
  if (!is_type(type) || !x) return GARFIELD_EINVAL;
  garfield_status st = check_size(tokens, outputs);
  if (st == GARFIELD_OK) st = check_size(tokens, x->cols);
  if (st == GARFIELD_OK) st = check_size(outputs, x->cols);
  if (st == GARFIELD_OK) st = check_counts(n, counts, tokens);
  if (st != GARFIELD_OK) return st;
  if (outputs > kMaxOutputs || x->ld_values > kMaxStride || x->ld_exponents > kMaxStride)
    return GARFIELD_ETOOBIG;
  const int64_t length = outputs * x->cols;
  if (!matrix_ok(dy, type, tokens, outputs, lddy) || !block8_ok(x, tokens, x->cols) ||
      (length > 0 && !dw) || !gradient_ok(dw, n, length, ld_dw) ||
      !gradient_ok(dbias, n, outputs, ld_dbias))
    return GARFIELD_EINVAL;
  if (!workspace_ok(workspace, workspace_bytes,
                    weight_gradient_bytes(type, tokens, outputs, x->cols, dy, lddy, n, counts)))
    return GARFIELD_EINVAL;
  if (outputs == 0) return GARFIELD_OK;
  WeightGradient a = {};
  a.dy = dy;
  a.type = type;
  a.tokens = tokens;
  a.outputs = outputs;
  a.lddy = lddy;
  a.x = *x;
  a.n = n;
  a.counts = counts;
  a.dw = dw;
  a.ld_dw = ld_dw;
  a.dbias = dbias;
  a.ld_dbias = ld_dbias;
  return status_of(enqueue_weight_gradient(a, workspace, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
