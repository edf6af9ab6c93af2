// Internal declarations of the worker's operators (see garfield_worker.h for
// what each computes). Arguments are checked by worker_api.cpp.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "garfield_worker.h"

namespace garfield {

constexpr int kWorkersMax = GARFIELD_NMAX;

// The workers' tokens, cut into chunks of at most `rows` tokens of one worker.
// Passed to kernels by value.
struct Chunks {
  int n = 0;
  int64_t rows = 0;
  int64_t token0[kWorkersMax + 1] = {};  // first token of each worker
  int chunk0[kWorkersMax + 1] = {};      // first chunk of each worker
};
Chunks make_chunks(int n, const int64_t* counts, int64_t rows);

hipError_t enqueue_checkpoint(const void* x, int type, int64_t rows, int64_t cols, int64_t ld,
                              bool transposed, const garfield_block8& out, hipStream_t s);
hipError_t enqueue_restore(const garfield_block8& c, void* out, int type, int64_t ld,
                           hipStream_t s);

struct LayerNorm {
  int64_t rows, cols;
  const void *x, *weight, *bias;
  int64_t ldx;
  bool weight_f32;  // weight and bias are fp32; else of x's type
  float eps;
  double share;  // 1 / cols
  void* y;
  int64_t ldy;
  float *mean, *rstd;
  garfield_block8 y8, x8;  // values null: not asked for
};
hipError_t enqueue_layernorm(const LayerNorm& a, int type, hipStream_t s);

struct LayerNormBackward {
  int64_t rows, cols;
  const void *dy, *x, *weight;
  int64_t lddy, ldx;
  garfield_block8 x8;  // where x is null
  bool weight_f32;
  const float *mean, *rstd;
  void* dx;
  int64_t lddx;
  float *dweight, *dbias;
  int64_t ld_dweight, ld_dbias;
};
Chunks layernorm_backward_chunks(int64_t rows, int64_t cols, int n, const int64_t* counts);
size_t layernorm_backward_bytes(const Chunks& c, int64_t cols);
hipError_t enqueue_layernorm_backward(const LayerNormBackward& a, int type, const Chunks& c,
                                      void* workspace, hipStream_t s);

size_t linear8_bytes(int64_t tokens, int64_t outputs, int64_t inputs);
hipError_t enqueue_linear8(const garfield_block8& x, const garfield_block8& w, const float* bias,
                           bool fast, void* out, int type, int64_t ld, void* workspace, hipStream_t s);

struct WeightGradient {
  const void* dy;
  int type;
  int64_t tokens, outputs, lddy;
  garfield_block8 x;
  int n;
  const int64_t* counts;
  float* dw;
  int64_t ld_dw;
  float* dbias;
  int64_t ld_dbias;
};
size_t weight_gradient_bytes(int type, int64_t tokens, int64_t outputs, int64_t inputs,
                             const void* dy, int64_t lddy, int n, const int64_t* counts);
hipError_t enqueue_weight_gradient(const WeightGradient& a, void* workspace, hipStream_t s);

}  // namespace garfield
