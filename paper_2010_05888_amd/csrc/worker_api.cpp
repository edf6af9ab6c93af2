// C-ABI of the worker's operators: argument validation and dispatch. See
// include/garfield_worker.h.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

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
// Dense products address 256 rows of a matrix with 32 bits.
constexpr int64_t kMaxDense = int64_t{1} << 20;
constexpr int kMaxTensors = 1 << 20;
constexpr int64_t kMaxLength = int64_t{1} << 34;

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

bool is_activation(int a) { return a >= GARFIELD_NO_ACTIVATION && a <= GARFIELD_SILU; }

garfield_status check_product(int64_t rows, int64_t cols, int64_t depth) {
  garfield_status st = check_size(rows, depth);
  if (st == GARFIELD_OK) st = check_size(cols, depth);
  if (st == GARFIELD_OK) st = check_size(rows, cols);
  return st == GARFIELD_OK && (cols > kMaxDense || depth > kMaxDense) ? GARFIELD_ETOOBIG : st;
}

Product forward_product(const void* x, int type, int64_t tokens, int64_t inputs, int64_t ldx,
                        const void* w, int64_t outputs, int64_t ldw) {
  Product p;
  p.type = type;
  p.rows = tokens;
  p.cols = outputs;
  p.depth = inputs;
  p.a = {x, ldx, false};
  p.b = {w, ldw, false};
  return p;
}

Product backward_product(const void* dy, int type, int64_t tokens, int64_t outputs, int64_t lddy,
                         const void* w, int64_t inputs, int64_t ldw) {
  Product p;
  p.type = type;
  p.rows = tokens;
  p.cols = inputs;
  p.depth = outputs;
  p.a = {dy, lddy, false};
  p.b = {w, ldw, true};
  return p;
}

DenseGradient dense_gradient(const void* dy, int type, int64_t tokens, int64_t outputs,
                             int64_t lddy, const void* x, int64_t inputs, int64_t ldx, int n,
                             const int64_t* counts) {
  DenseGradient a = {};
  a.dy = dy;
  a.x = x;
  a.type = type;
  a.tokens = tokens;
  a.outputs = outputs;
  a.inputs = inputs;
  a.lddy = lddy;
  a.ldx = ldx;
  a.n = n;
  a.counts = counts;
  return a;
}

garfield_status check_dense_gradient(int type, int64_t tokens, int64_t outputs, int64_t inputs,
                                     int n, const int64_t* counts) {
  if (!is_type(type)) return GARFIELD_EINVAL;
  garfield_status st = check_size(tokens, outputs);
  if (st == GARFIELD_OK) st = check_size(tokens, inputs);
  if (st == GARFIELD_OK) st = check_size(outputs, inputs);
  if (st == GARFIELD_OK) st = check_counts(n, counts, tokens);
  if (st == GARFIELD_OK && (outputs > kMaxDense || inputs > kMaxDense)) return GARFIELD_ETOOBIG;
  return st;
}

garfield_status check_block(const garfield_residual_block* b) {
  if (!b || !is_type(b->type) || (b->wtype != GARFIELD_F32 && b->wtype != b->type))
    return GARFIELD_EINVAL;
  const garfield_status st = check_size(b->rows, b->cols);
  if (st != GARFIELD_OK) return st;
  const int64_t bytes = element_bytes(b->wtype);
  auto parameter = [&](const void* p) { return !p || vector_ok(p, bytes, b->cols); };
  if (b->cols == 0 || !(b->eps >= 0.0f) || !parameter(b->weight) || !parameter(b->bias) ||
      !parameter(b->post_weight) || !parameter(b->post_bias) || (b->bias && !b->weight) ||
      (b->post_bias && !b->post_weight) || (b->rms && (b->bias || b->post_bias)))
    return GARFIELD_EINVAL;
  if (b->gate && (b->ld_gate == 0 ? !parameter(b->gate)
                                  : !matrix_ok(b->gate, b->type, b->rows, b->cols, b->ld_gate)))
    return GARFIELD_EINVAL;
  return GARFIELD_OK;
}

garfield_status check_tensors(const garfield_gradient* t, int count, int n) {
  if (count < 0 || n < 1 || (count > 0 && !t)) return GARFIELD_EINVAL;
  if (n > GARFIELD_NMAX || count > kMaxTensors) return GARFIELD_ETOOBIG;
  for (int i = 0; i < count; ++i) {
    if (!is_type(t[i].type) || t[i].length < 0) return GARFIELD_EINVAL;
    if (t[i].length > kMaxLength) return GARFIELD_ETOOBIG;
  }
  return GARFIELD_OK;
}

bool tensors_ok(const garfield_gradient* t, int count, int n) {
  for (int i = 0; i < count; ++i)
    if (t[i].length > 0 && (!t[i].values || !aligned(t[i].values, element_bytes(t[i].type)) ||
                            (n > 1 && t[i].ld < t[i].length)))
      return false;
  return true;
}

// A tensor's bytes: n rows of `length`, `apart` apart.
struct Range {
  uintptr_t first, end;
  uintptr_t apart, length;
};
Range range_of(const garfield_gradient& t, int n) {
  const uintptr_t b = element_bytes(t.type), p = reinterpret_cast<uintptr_t>(t.values);
  const uintptr_t apart = n > 1 ? t.ld * b : 0, length = t.length * b;
  return {p, p + apart * (n - 1) + length, apart, length};
}

// Whether no two of the tensors have a byte in common. Tensors whose ranges overlap may still
// be columns of one matrix: rows equally far apart, and no columns shared.
bool ranges_apart(std::vector<Range>& all, int n) {
  std::sort(all.begin(), all.end(), [](const Range& x, const Range& y) { return x.first < y.first; });
  // In a group of ranges that overlap, all must be columns of the first one's matrix: its
  // rows, in which no column starts before the last one's end, and which wrap round once.
  for (size_t i = 0; i < all.size();) {
    const Range& r = all[i];
    uintptr_t end = r.end, used = r.length;
    size_t k = i + 1;
    for (; k < all.size() && all[k].first < end; ++k) {
      const uintptr_t at = all[k].first - r.first;
      if (n == 1 || all[k].apart != r.apart || at < used || at + all[k].length > r.apart) return false;
      used = at + all[k].length;
      end = std::max(end, all[k].end);
    }
    i = k;
  }
  return true;
}

bool tensors_apart(const garfield_gradient* t, int count, int n) {
  std::vector<Range> all;
  all.reserve(count);
  for (int i = 0; i < count; ++i)
    if (t[i].length > 0) all.push_back(range_of(t[i], n));
  return ranges_apart(all, n);
}

// Whether none of them has a byte in common with the rows that are written.
bool apart_from(const garfield_gradient* t, int count, int n, float* out, int64_t d, int64_t ld) {
  const garfield_gradient rows = {out, d, ld, GARFIELD_F32};
  const Range to = range_of(rows, n);
  std::vector<Range> both(2);
  for (int i = 0; i < count; ++i) {
    if (t[i].length == 0) continue;
    const Range r = range_of(t[i], n);
    if (r.end <= to.first || to.end <= r.first) continue;
    both[0] = r;
    both[1] = to;
    if (!ranges_apart(both, n)) return false;
  }
  return true;
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

size_t garfield_linear_workspace(const void* x, int type, int64_t tokens, int64_t inputs,
                                 int64_t ldx, const void* w, int64_t outputs, int64_t ldw) {
  if (!is_type(type) || check_product(tokens, outputs, inputs) != GARFIELD_OK) return 0;
  return product_bytes(forward_product(x, type, tokens, inputs, ldx, w, outputs, ldw));
}

garfield_status garfield_linear(const void* x, int type, int64_t tokens, int64_t inputs,
                                int64_t ldx, const void* w, int64_t outputs, int64_t ldw,
                                const void* bias, int btype, int activation, const void* residual,
                                int64_t ld_residual, void* out, int64_t ld_out, void* pre,
                                int64_t ld_pre, void* workspace, size_t workspace_bytes,
                                void* stream) {
  if (!is_type(type) || (bias && btype != GARFIELD_F32 && btype != type) ||
      !is_activation(activation))
    return GARFIELD_EINVAL;
  const garfield_status st = check_product(tokens, outputs, inputs);
  if (st != GARFIELD_OK) return st;
  if (!matrix_ok(x, type, tokens, inputs, ldx) || !matrix_ok(w, type, outputs, inputs, ldw) ||
      (bias && !vector_ok(bias, element_bytes(btype), outputs)) ||
      (residual && !matrix_ok(residual, type, tokens, outputs, ld_residual)) ||
      !matrix_ok(out, type, tokens, outputs, ld_out) ||
      (pre && !matrix_ok(pre, type, tokens, outputs, ld_pre)))
    return GARFIELD_EINVAL;
  Product p = forward_product(x, type, tokens, inputs, ldx, w, outputs, ldw);
  if (!workspace_ok(workspace, workspace_bytes, product_bytes(p))) return GARFIELD_EINVAL;
  if (tokens == 0 || outputs == 0) return GARFIELD_OK;
  p.to.bias = bias;
  p.to.bias_f32 = btype == GARFIELD_F32;
  p.to.activation = activation;
  p.to.residual = residual;
  p.to.ld_residual = ld_residual;
  p.to.out = out;
  p.to.ld_out = ld_out;
  p.to.pre = pre;
  p.to.ld_pre = ld_pre;
  return status_of(enqueue_product(p, workspace, static_cast<hipStream_t>(stream)));
}

size_t garfield_linear_backward_workspace(const void* dy, int type, int64_t tokens,
                                          int64_t outputs, int64_t lddy, const void* w,
                                          int64_t inputs, int64_t ldw) {
  if (!is_type(type) || check_product(tokens, inputs, outputs) != GARFIELD_OK) return 0;
  return product_bytes(backward_product(dy, type, tokens, outputs, lddy, w, inputs, ldw));
}

garfield_status garfield_linear_backward(const void* dy, int type, int64_t tokens, int64_t outputs,
                                         int64_t lddy, const void* w, int64_t inputs, int64_t ldw,
                                         int activation, const void* pre, int64_t ld_pre,
                                         const void* residual, int64_t ld_residual, void* dx,
                                         int64_t lddx, void* workspace, size_t workspace_bytes,
                                         void* stream) {
  if (!is_type(type) || !is_activation(activation)) return GARFIELD_EINVAL;
  const garfield_status st = check_product(tokens, inputs, outputs);
  if (st != GARFIELD_OK) return st;
  if (!matrix_ok(dy, type, tokens, outputs, lddy) || !matrix_ok(w, type, outputs, inputs, ldw) ||
      (activation != GARFIELD_NO_ACTIVATION && !matrix_ok(pre, type, tokens, inputs, ld_pre)) ||
      (residual && !matrix_ok(residual, type, tokens, inputs, ld_residual)) ||
      !matrix_ok(dx, type, tokens, inputs, lddx))
    return GARFIELD_EINVAL;
  Product p = backward_product(dy, type, tokens, outputs, lddy, w, inputs, ldw);
  if (!workspace_ok(workspace, workspace_bytes, product_bytes(p))) return GARFIELD_EINVAL;
  if (tokens == 0 || inputs == 0) return GARFIELD_OK;
  p.to.activation = activation;
  p.to.before = activation != GARFIELD_NO_ACTIVATION ? pre : nullptr;
  p.to.ld_before = ld_pre;
  p.to.residual = residual;
  p.to.ld_residual = ld_residual;
  p.to.out = dx;
  p.to.ld_out = lddx;
  return status_of(enqueue_product(p, workspace, static_cast<hipStream_t>(stream)));
}

garfield_status garfield_activation_backward(const void* dy, int type, int64_t rows, int64_t cols,
                                             int64_t lddy, int activation, const void* pre,
                                             int64_t ld_pre, void* dp, int64_t lddp,
                                             void* stream) {
  if (!is_type(type) || !is_activation(activation)) return GARFIELD_EINVAL;
  const garfield_status st = check_size(rows, cols);
  if (st != GARFIELD_OK) return st;
  if (!matrix_ok(dy, type, rows, cols, lddy) || !matrix_ok(pre, type, rows, cols, ld_pre) ||
      !matrix_ok(dp, type, rows, cols, lddp))
    return GARFIELD_EINVAL;
  if (rows == 0 || cols == 0) return GARFIELD_OK;
  return status_of(enqueue_activation_backward(dy, lddy, pre, ld_pre, activation, dp, lddp, type,
                                               rows, cols, static_cast<hipStream_t>(stream)));
}

size_t garfield_linear_weight_gradient_workspace(const void* dy, int type, int64_t tokens,
                                                 int64_t outputs, int64_t lddy, const void* x,
                                                 int64_t inputs, int64_t ldx, int n,
                                                 const int64_t* counts) {
  if (check_dense_gradient(type, tokens, outputs, inputs, n, counts) != GARFIELD_OK) return 0;
  return dense_gradient_bytes(
      dense_gradient(dy, type, tokens, outputs, lddy, x, inputs, ldx, n, counts));
}

garfield_status garfield_linear_weight_gradient(const void* dy, int type, int64_t tokens,
                                                int64_t outputs, int64_t lddy, const void* x,
                                                int64_t inputs, int64_t ldx, int n,
                                                const int64_t* counts, float* dw, int64_t ld_dw,
                                                float* dbias, int64_t ld_dbias, void* workspace,
                                                size_t workspace_bytes, void* stream) {
  const garfield_status st = check_dense_gradient(type, tokens, outputs, inputs, n, counts);
  if (st != GARFIELD_OK) return st;
  const int64_t length = outputs * inputs;
  if (!matrix_ok(dy, type, tokens, outputs, lddy) || !matrix_ok(x, type, tokens, inputs, ldx) ||
      (length > 0 && !dw) || !gradient_ok(dw, n, length, ld_dw) ||
      !gradient_ok(dbias, n, outputs, ld_dbias))
    return GARFIELD_EINVAL;
  DenseGradient a = dense_gradient(dy, type, tokens, outputs, lddy, x, inputs, ldx, n, counts);
  if (!workspace_ok(workspace, workspace_bytes, dense_gradient_bytes(a))) return GARFIELD_EINVAL;
  if (outputs == 0) return GARFIELD_OK;
  a.dw = dw;
  a.ld_dw = ld_dw;
  a.dbias = dbias;
  a.ld_dbias = ld_dbias;
  return status_of(enqueue_dense_gradient(a, workspace, static_cast<hipStream_t>(stream)));
}

garfield_status garfield_residual_norm(const garfield_residual_block* b, const void* x,
                                       int64_t ldx, const void* h, int64_t ldh, void* s,
                                       int64_t lds, void* y, int64_t ldy, float* mean, float* rstd,
                                       float* post_mean, float* post_rstd,
                                       const garfield_block8* y8, void* stream) {
  const garfield_status st = check_block(b);
  if (st != GARFIELD_OK) return st;
  const int64_t rows = b->rows, cols = b->cols;
  auto stats_ok = [&](const void* norm, float* m, float* r) {
    return !norm || (vector_ok(r, 4, rows) && (b->rms || vector_ok(m, 4, rows)));
  };
  if (!matrix_ok(x, b->type, rows, cols, ldx) || !matrix_ok(h, b->type, rows, cols, ldh) ||
      !matrix_ok(s, b->type, rows, cols, lds) || (y && !matrix_ok(y, b->type, rows, cols, ldy)) ||
      (!b->weight && (y || y8)) || !stats_ok(b->weight, mean, rstd) ||
      !stats_ok(b->post_weight, post_mean, post_rstd) || (y8 && !block8_ok(y8, rows, cols)))
    return GARFIELD_EINVAL;
  if (rows == 0) return GARFIELD_OK;
  ResidualNorm a = {};
  a.b = *b;
  a.x = x;
  a.h = h;
  a.ldx = ldx;
  a.ldh = ldh;
  a.share = 1.0 / static_cast<double>(cols);
  a.s = s;
  a.y = y;
  a.lds = lds;
  a.ldy = ldy;
  a.mean = mean;
  a.rstd = rstd;
  a.post_mean = post_mean;
  a.post_rstd = post_rstd;
  if (y8) a.y8 = *y8;
  return status_of(enqueue_residual_norm(a, static_cast<hipStream_t>(stream)));
}

size_t garfield_residual_norm_backward_workspace(const garfield_residual_block* b, int n,
                                                 const int64_t* counts) {
  if (check_block(b) != GARFIELD_OK || check_counts(n, counts, b->rows) != GARFIELD_OK) return 0;
  return residual_norm_backward_bytes(*b, residual_norm_backward_chunks(*b, n, counts));
}

garfield_status garfield_residual_norm_backward(
    const garfield_residual_block* b, const void* ds, int64_t ldds, const void* dy, int64_t lddy,
    const void* s, int64_t lds, const void* h, int64_t ldh, const float* mean, const float* rstd,
    const float* post_mean, const float* post_rstd, void* dx, int64_t lddx, void* dh,
    int64_t lddh, void* dgate, int64_t lddgate, int n, const int64_t* counts,
    const garfield_residual_gradients* gradients, void* workspace, size_t workspace_bytes,
    void* stream) {
  garfield_status st = check_block(b);
  if (st == GARFIELD_OK) st = check_counts(n, counts, b->rows);
  if (st != GARFIELD_OK) return st;
  const int64_t rows = b->rows, cols = b->cols;
  auto given = [&](const void* p, int64_t ld) { return matrix_ok(p, b->type, rows, cols, ld); };
  auto stats_ok = [&](const float* m, const float* r) {
    return vector_ok(r, 4, rows) && (b->rms || vector_ok(m, 4, rows));
  };
  const garfield_residual_gradients to = gradients ? *gradients : garfield_residual_gradients{};
  const bool by_tokens = b->gate && b->ld_gate != 0;
  if ((!ds && !dy && rows > 0) || (ds && !given(ds, ldds)) ||
      (dy && (!b->weight || !given(dy, lddy) || !given(s, lds) || !stats_ok(mean, rstd))) ||
      !given(h, ldh) || (b->post_weight && !stats_ok(post_mean, post_rstd)) ||
      (dx && !given(dx, lddx)) || (dh && !given(dh, lddh)) ||
      (dgate && (!by_tokens || !given(dgate, lddgate))) ||
      (to.weight && !b->weight) || (to.bias && (!b->weight || b->rms)) ||
      (to.post_weight && !b->post_weight) || (to.post_bias && (!b->post_weight || b->rms)) ||
      (to.gate && (!b->gate || by_tokens)) || !gradient_ok(to.weight, n, cols, to.ld_weight) ||
      !gradient_ok(to.bias, n, cols, to.ld_bias) ||
      !gradient_ok(to.post_weight, n, cols, to.ld_post_weight) ||
      !gradient_ok(to.post_bias, n, cols, to.ld_post_bias) ||
      !gradient_ok(to.gate, n, cols, to.ld_gate))
    return GARFIELD_EINVAL;
  const Chunks chunks = residual_norm_backward_chunks(*b, n, counts);
  if (!workspace_ok(workspace, workspace_bytes, residual_norm_backward_bytes(*b, chunks)))
    return GARFIELD_EINVAL;
  ResidualNormBackward a = {};
  a.b = *b;
  a.ds = ds;
  a.dy = dy;
  a.s = s;
  a.h = h;
  a.ldds = ldds;
  a.lddy = lddy;
  a.lds = lds;
  a.ldh = ldh;
  a.mean = mean;
  a.rstd = rstd;
  a.post_mean = post_mean;
  a.post_rstd = post_rstd;
  a.dx = dx;
  a.dh = dh;
  a.dgate = dgate;
  a.lddx = lddx;
  a.lddh = lddh;
  a.lddgate = lddgate;
  a.to = to;
  return status_of(
      enqueue_residual_norm_backward(a, chunks, workspace, static_cast<hipStream_t>(stream)));
}

size_t garfield_clip_workspace(const garfield_gradient* tensors, int count, int n) {
  if (check_tensors(tensors, count, n) != GARFIELD_OK) return 0;
  return clip_bytes(tensors, count, n);
}

garfield_status garfield_gradient_norms(const garfield_gradient* tensors, int count, int n,
                                        float* norms, void* workspace, size_t workspace_bytes,
                                        void* stream) {
  const garfield_status st = check_tensors(tensors, count, n);
  if (st != GARFIELD_OK) return st;
  if (!tensors_ok(tensors, count, n) || !vector_ok(norms, 4, n) ||
      !workspace_ok(workspace, workspace_bytes, clip_bytes(tensors, count, n)))
    return GARFIELD_EINVAL;
  return status_of(enqueue_clip(tensors, count, n, NAN, norms, nullptr, 0, workspace,
                                static_cast<hipStream_t>(stream)));
}

garfield_status garfield_clip_gradients(const garfield_gradient* tensors, int count, int n,
                                        float max_norm, float* norms, float* out, int64_t ld_out,
                                        void* workspace, size_t workspace_bytes, void* stream) {
  const garfield_status st = check_tensors(tensors, count, n);
  if (st != GARFIELD_OK) return st;
  if (!(max_norm >= 0.0f)) return GARFIELD_EINVAL;
  int64_t d = 0;
  for (int i = 0; i < count; ++i) d += tensors[i].length;
  if (d > kMaxLength) return GARFIELD_ETOOBIG;
  if (!tensors_ok(tensors, count, n) || !vector_ok(norms, 4, n) || !gradient_ok(out, n, d, ld_out) ||
      !workspace_ok(workspace, workspace_bytes, clip_bytes(tensors, count, n)))
    return GARFIELD_EINVAL;
  try {
    if (out ? !apart_from(tensors, count, n, out, d, ld_out) : !tensors_apart(tensors, count, n))
      return GARFIELD_EINVAL;
  } catch (const std::bad_alloc&) {
    return GARFIELD_ENOMEM;
  }
  return status_of(enqueue_clip(tensors, count, n, max_norm, norms, out, ld_out, workspace,
                                static_cast<hipStream_t>(stream)));
}

}  // extern "C"
