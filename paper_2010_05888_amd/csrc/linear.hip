// Products of 16- and 32-bit matrices with an epilogue: a linear layer's forward pass, the
// gradient of its input, and of each worker the gradient of its weights.

#include "activation.h"
#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

// One output of the epilogue.
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t m, int64_t j, float v) {
  if (e.before) {
    v *= slope(e.activation, static_cast<float>(static_cast<const T*>(e.before)[m * e.ld_before + j]));
  } else {
    if (e.bias)
      v += e.bias_f32 ? static_cast<const float*>(e.bias)[j]
                      : static_cast<float>(static_cast<const T*>(e.bias)[j]);
    if (e.pre) static_cast<T*>(e.pre)[m * e.ld_pre + j] = static_cast<T>(v);
    v = activate(e.activation, v);
  }
  if (e.residual) v += static_cast<float>(static_cast<const T*>(e.residual)[m * e.ld_residual + j]);
  static_cast<T*>(e.out)[m * e.ld_out + j] = static_cast<T>(v);
}

// sum[4][4] of a tile of 64 x 64 outputs: thread t has rows t / 16 * 4 on and columns
// t % 16 * 4 on. Element (m, k) of A lies at a[m * am + k * ak], and B likewise.
template <typename T>
__device__ __forceinline__ void tile_sums(const T* a, int64_t am, int64_t ak, int64_t rows,
                                          const T* b, int64_t bn, int64_t bk, int64_t cols,
                                          int64_t depth, int64_t m0, int64_t j0, float sum[4][4]) {
  __shared__ float as[16][64], bs[16][64];
  const int tm = threadIdx.x / 16 * 4, tj = threadIdx.x % 16 * 4;
  for (int64_t k0 = 0; k0 < depth; k0 += 16) {
    __syncthreads();
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int64_t am_ = ak == 1 ? i / 16 : i % 64, ak_ = ak == 1 ? i % 16 : i / 64;
      as[ak_][am_] = m0 + am_ < rows && k0 + ak_ < depth
                         ? static_cast<float>(a[(m0 + am_) * am + (k0 + ak_) * ak]) : 0.0f;
      const int64_t bn_ = bk == 1 ? i / 16 : i % 64, bk_ = bk == 1 ? i % 16 : i / 64;
      bs[bk_][bn_] = j0 + bn_ < cols && k0 + bk_ < depth
                         ? static_cast<float>(b[(j0 + bn_) * bn + (k0 + bk_) * bk]) : 0.0f;
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int i = 0; i < 4; ++i)
        for (int c = 0; c < 4; ++c)
          sum[i][c] = __builtin_fmaf(as[k][tm + i], bs[k][tj + c], sum[i][c]);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_product(Product p, uint32_t tiles_j) {
  const int64_t m0 = blockIdx.x / tiles_j * int64_t{64}, j0 = blockIdx.x % tiles_j * int64_t{64};
  float sum[4][4] = {};
  tile_sums<T>(static_cast<const T*>(p.a.p), p.a.across ? 1 : p.a.ld, p.a.across ? p.a.ld : 1,
               p.rows, static_cast<const T*>(p.b.p), p.b.across ? 1 : p.b.ld,
               p.b.across ? p.b.ld : 1, p.cols, p.depth, m0, j0, sum);
  for (int i = 0; i < 4; ++i)
    for (int c = 0; c < 4; ++c) {
      const int64_t m = m0 + threadIdx.x / 16 * 4 + i, j = j0 + threadIdx.x % 16 * 4 + c;
      if (m < p.rows && j < p.cols) finish<T>(p.to, m, j, sum[i][c]);
    }
}

struct Workers {
  int64_t first[kWorkersMax + 1];
};

template <typename T>
__global__ __launch_bounds__(256) void k_dense_gradient(DenseGradient a, Workers w,
                                                        uint32_t tiles_k) {
  const int64_t j0 = blockIdx.x / tiles_k * int64_t{64}, k0 = blockIdx.x % tiles_k * int64_t{64};
  const int64_t t0 = w.first[blockIdx.y], tokens = w.first[blockIdx.y + 1] - t0;
  float sum[4][4] = {};
  tile_sums<T>(static_cast<const T*>(a.dy) + t0 * a.lddy, 1, a.lddy, a.outputs,
               static_cast<const T*>(a.x) + t0 * a.ldx, 1, a.ldx, a.inputs, tokens, j0, k0, sum);
  for (int i = 0; i < 4; ++i)
    for (int c = 0; c < 4; ++c) {
      const int64_t j = j0 + threadIdx.x / 16 * 4 + i, k = k0 + threadIdx.x % 16 * 4 + c;
      if (j < a.outputs && k < a.inputs)
        a.dw[blockIdx.y * a.ld_dw + j * a.inputs + k] = sum[i][c];
    }
}

template <typename T>
__global__ __launch_bounds__(64) void k_dense_bias(DenseGradient a, Workers w) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;
  if (j >= a.outputs) return;
  float sum = 0.0f;
  for (int64_t t = w.first[blockIdx.y]; t < w.first[blockIdx.y + 1]; ++t)
    sum += static_cast<float>(static_cast<const T*>(a.dy)[t * a.lddy + j]);
  a.dbias[blockIdx.y * a.ld_dbias + j] = sum;
}

// Eight values a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_activation_backward(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ pre, int64_t ld_pre,
    int activation, T* __restrict__ dp, int64_t lddp, int64_t rows, int64_t cols) {
  const int64_t vectors = (cols + 7) / 8;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < rows * vectors;
       i += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t m = i / vectors, c = i % vectors * 8;
    float g[8], p[8];
    load8_upto(dy + m * lddy + c, cols - c, g);
    load8_upto(pre + m * ld_pre + c, cols - c, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) g[e] *= slope(activation, p[e]);
    store8_upto(dp + m * lddp + c, cols - c, g);
  }
}

template <typename T>
void launch_product(const Product& p, hipStream_t s) {
  const uint32_t tiles_j = static_cast<uint32_t>((p.cols + 63) / 64);
  launch("product", k_product<T>, dim3(static_cast<uint32_t>((p.rows + 63) / 64) * tiles_j),
         dim3(256), 0, s, p, tiles_j);
}

template <typename T>
void launch_gradient(const DenseGradient& a, hipStream_t s) {
  Workers w = {};
  for (int i = 0; i < a.n; ++i) w.first[i + 1] = w.first[i] + a.counts[i];
  const uint32_t tiles_k = static_cast<uint32_t>((a.inputs + 63) / 64);
  const uint32_t tiles_j = static_cast<uint32_t>((a.outputs + 63) / 64);
  if (a.inputs > 0)
    launch("dense_gradient", k_dense_gradient<T>, dim3(tiles_j * tiles_k, a.n), dim3(256), 0, s, a,
           w, tiles_k);
  if (a.dbias) launch("dense_bias", k_dense_bias<T>, dim3(tiles_j, a.n), dim3(64), 0, s, a, w);
}

}  // namespace

size_t product_bytes(const Product&) { return 0; }

hipError_t enqueue_product(const Product& p, void*, hipStream_t s) {
  if (p.type == GARFIELD_F32) launch_product<float>(p, s);
  else if (p.type == GARFIELD_BF16) launch_product<__bf16>(p, s);
  else launch_product<_Float16>(p, s);
  return hipGetLastError();
}

size_t dense_gradient_bytes(const DenseGradient&) { return 0; }

hipError_t enqueue_dense_gradient(const DenseGradient& a, void*, hipStream_t s) {
  if (a.type == GARFIELD_F32) launch_gradient<float>(a, s);
  else if (a.type == GARFIELD_BF16) launch_gradient<__bf16>(a, s);
  else launch_gradient<_Float16>(a, s);
  return hipGetLastError();
}

template <typename T>
static void launch_slope(const void* dy, int64_t lddy, const void* pre, int64_t ld_pre,
                         int activation, void* dp, int64_t lddp, int64_t rows, int64_t cols,
                         hipStream_t s) {
  const int64_t groups = (rows * ((cols + 7) / 8) + kBlock - 1) / kBlock, most = int64_t{1} << 23;
  launch("activation_backward", k_activation_backward<T>,
         dim3(static_cast<uint32_t>(groups < most ? groups : most)), dim3(kBlock), 0, s,
         static_cast<const T*>(dy), lddy, static_cast<const T*>(pre), ld_pre, activation,
         static_cast<T*>(dp), lddp, rows, cols);
}

hipError_t enqueue_activation_backward(const void* dy, int64_t lddy, const void* pre,
                                       int64_t ld_pre, int activation, void* dp, int64_t lddp,
                                       int type, int64_t rows, int64_t cols, hipStream_t s) {
  if (type == GARFIELD_F32)
    launch_slope<float>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  else if (type == GARFIELD_BF16)
    launch_slope<__bf16>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  else
    launch_slope<_Float16>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  return hipGetLastError();
}

}  // namespace garfield
