// The residual around a block with the norms before and after it, and its backward pass with
// the parameters' gradients of each worker.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

template <typename F>
__device__ __forceinline__ F sum_group(F v, F* at) {
  v = sum_wave(v);
  __syncthreads();  // the last sum has been read
  if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
  __syncthreads();
  v = 0;
#pragma unroll
  for (int w = 0; w < kBlock / 64; ++w) v += at[w];
  return v;
}

template <typename T>
__device__ __forceinline__ void load_parameter(const void* p, bool f32, int64_t c, int64_t left,
                                               float missing, float* v) {
  if (!p) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = missing;
  } else if (f32) {
    load8_upto(static_cast<const float*>(p) + c, left, v);
  } else {
    load8_upto(static_cast<const T*>(p) + c, left, v);
  }
}

template <typename T>
__device__ __forceinline__ void load_gate(const garfield_residual_block& b, int64_t row, int64_t c,
                                          float* v) {
  if (b.gate && b.ld_gate)
    load8_upto(static_cast<const T*>(b.gate) + row * b.ld_gate + c, b.cols - c, v);
  else
    load_parameter<T>(b.gate, b.wtype == GARFIELD_F32, c, b.cols - c, 1.0f, v);
}

// N_post(h) of eight columns; hat is what the weight multiplies.
template <typename T>
__device__ __forceinline__ void post_norm(const garfield_residual_block& b, const float* h,
                                          float mean, float rstd, int64_t c, float* hat, float* f) {
  float w[8], bias[8];
  const bool f32 = b.wtype == GARFIELD_F32;
  load_parameter<T>(b.post_weight, f32, c, b.cols - c, 1.0f, w);
  load_parameter<T>(b.post_bias, f32, c, b.cols - c, 0.0f, bias);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    hat[e] = (h[e] - mean) * rstd;
    f[e] = b.post_weight ? __builtin_fmaf(hat[e], w[e], bias[e]) : h[e];
  }
}

template <typename T>
__device__ __forceinline__ void stream_values(const ResidualNorm& a, int64_t row, int64_t c,
                                              float mean, float rstd, float* v) {
  float h[8], hat[8], f[8], g[8];
  const int64_t left = a.b.cols - c;
  load8_upto(static_cast<const T*>(a.h) + row * a.ldh + c, left, h);
  load8_upto(static_cast<const T*>(a.x) + row * a.ldx + c, left, v);
  post_norm<T>(a.b, h, mean, rstd, c, hat, f);
  load_gate<T>(a.b, row, c, g);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(a.b.scale, v[e], g[e] * f[e]);
}

// Mean (0 with rms) and 1 / deviation of a row, `values` giving eight columns of it.
template <typename F>
__device__ __forceinline__ void statistics(const garfield_residual_block& b, double share,
                                           double* totals, float* sums, F&& values, float* mean,
                                           float* rstd) {
  float v[8];
  *mean = 0.0f;
  if (!b.rms) {
    double sum = 0.0;
    for (int64_t c = threadIdx.x * 8; c < b.cols; c += kBlock * 8) {
      values(c, v);
      for (int e = 0; e < 8 && c + e < b.cols; ++e) sum += v[e];
    }
    *mean = static_cast<float>(sum_group(sum, totals) * share);
  }
  float square = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kBlock * 8) {
    values(c, v);
    for (int e = 0; e < 8 && c + e < b.cols; ++e)
      square = __builtin_fmaf(v[e] - *mean, v[e] - *mean, square);
  }
  *rstd = 1.0f / __builtin_sqrtf(sum_group(square, sums) * static_cast<float>(share) + b.eps);
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_residual_norm(ResidualNorm a) {
  __shared__ double totals[kBlock / 64];
  __shared__ float sums[kBlock / 64];
  const int64_t row = blockIdx.x;
  float pm = 0.0f, pr = 1.0f, mean, rstd, v[8];
  if (a.b.post_weight) {
    statistics(a.b, a.share, totals, sums, [&](int64_t c, float* h) {
      load8_upto(static_cast<const T*>(a.h) + row * a.ldh + c, a.b.cols - c, h);
    }, &pm, &pr);
    if (threadIdx.x == 0) {
      if (!a.b.rms) a.post_mean[row] = pm;
      a.post_rstd[row] = pr;
    }
  }
  auto values = [&](int64_t c, float* t) { stream_values<T>(a, row, c, pm, pr, t); };
  if (a.b.weight) {
    statistics(a.b, a.share, totals, sums, values, &mean, &rstd);
    if (threadIdx.x == 0) {
      if (!a.b.rms) a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
  }
  const bool f32 = a.b.wtype == GARFIELD_F32;
  const int64_t padded = (a.b.cols + 511) / 512 * 512;
  for (int64_t c = threadIdx.x * 8; c < padded; c += kBlock * 8) {
    const int64_t left = a.b.cols - c;
    float w[8], bias[8];
    if (left > 0) {
      values(c, v);
      store8_upto(static_cast<T*>(a.s) + row * a.lds + c, left, v);
    }
    if (!a.b.weight) continue;
    load_parameter<T>(a.b.weight, f32, c, left, 1.0f, w);
    load_parameter<T>(a.b.bias, f32, c, left, 0.0f, bias);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = e < left ? __builtin_fmaf((v[e] - mean) * rstd, w[e], bias[e]) : 0.0f;
    if (a.y && left > 0) store8_upto(static_cast<T*>(a.y) + row * a.ldy + c, left, v);
    if (a.y8.values) {
      const int s = block_shift(max16(largest<8>(v)));
      const int64_t blocks = (a.y8.cols + kBlock8 - 1) / kBlock8, k = c / kBlock8;
      if (k < blocks)
        *reinterpret_cast<u2*>(a.y8.values + row * a.y8.ld_values + c) = encode8(v, s);
      if (c % kBlock8 == 0 && k < (blocks + 3) / 4 * 4)
        a.y8.exponents[row * a.y8.ld_exponents + k] = static_cast<uint8_t>(k < blocks ? s + 127 : 127);
    }
  }
}

// What the backward pass knows of eight columns of a row.
struct Eight {
  float g[8], df[8], post[8], f[8], hat[8], dy[8];
};

// g, df and dh's terms need along and across of both norms: given the first ones, 0 before.
template <typename T>
__device__ __forceinline__ void backward_values(const ResidualNormBackward& a, int64_t row,
                                                int64_t c, float along, float across, Eight& t) {
  const garfield_residual_block& b = a.b;
  const int64_t left = b.cols - c;
  const bool f32 = b.wtype == GARFIELD_F32;
  float w[8], h[8], gate[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t.g[e] = t.hat[e] = t.dy[e] = 0.0f;
  if (a.ds) load8_upto(static_cast<const T*>(a.ds) + row * a.ldds + c, left, t.g);
  if (a.dy) {
    load8_upto(static_cast<const T*>(a.dy) + row * a.lddy + c, left, t.dy);
    load8_upto(static_cast<const T*>(a.s) + row * a.lds + c, left, t.hat);
    load_parameter<T>(b.weight, f32, c, left, 1.0f, w);
    const float mean = b.rms ? 0.0f : a.mean[row], rstd = a.rstd[row];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t.hat[e] = (t.hat[e] - mean) * rstd;
      t.g[e] += rstd * (t.dy[e] * w[e] - along - t.hat[e] * across);
    }
  }
  load8_upto(static_cast<const T*>(a.h) + row * a.ldh + c, left, h);
  load_gate<T>(b, row, c, gate);
  post_norm<T>(b, h, b.post_weight && !b.rms ? a.post_mean[row] : 0.0f,
               b.post_weight ? a.post_rstd[row] : 1.0f, c, t.post, t.f);
#pragma unroll
  for (int e = 0; e < 8; ++e) t.df[e] = t.g[e] * gate[e];
}

// The means over a row of dy w (0 with rms) and dy w hat.
template <typename T>
__device__ __forceinline__ void backward_sums(const ResidualNormBackward& a, int64_t row,
                                              float* sums, float* along, float* across) {
  const garfield_residual_block& b = a.b;
  float x = 0.0f, y = 0.0f, w[8];
  Eight t;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kBlock * 8) {
    backward_values<T>(a, row, c, 0.0f, 0.0f, t);
    load_parameter<T>(b.weight, b.wtype == GARFIELD_F32, c, b.cols - c, 1.0f, w);
    for (int e = 0; e < 8 && c + e < b.cols; ++e) {
      x = __builtin_fmaf(t.dy[e], w[e], x);
      y = __builtin_fmaf(t.dy[e] * w[e], t.hat[e], y);
    }
  }
  const float cols = static_cast<float>(b.cols);
  *along = b.rms ? 0.0f : sum_group(x, sums) / cols;
  *across = sum_group(y, sums) / cols;
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_residual_dx(ResidualNormBackward a, float2* means) {
  __shared__ float sums[kBlock / 64];
  const garfield_residual_block& b = a.b;
  const int64_t row = blockIdx.x;
  float along = 0.0f, across = 0.0f, w[8];
  if (a.dy) backward_sums<T>(a, row, sums, &along, &across);
  if (threadIdx.x == 0) means[row] = {along, across};
  float x = 0.0f, y = 0.0f;
  Eight t;
  const bool f32 = b.wtype == GARFIELD_F32;
  if (b.post_weight) {
    for (int64_t c = threadIdx.x * 8; c < b.cols; c += kBlock * 8) {
      backward_values<T>(a, row, c, along, across, t);
      load_parameter<T>(b.post_weight, f32, c, b.cols - c, 1.0f, w);
      for (int e = 0; e < 8 && c + e < b.cols; ++e) {
        x = __builtin_fmaf(t.df[e], w[e], x);
        y = __builtin_fmaf(t.df[e] * w[e], t.post[e], y);
      }
    }
    const float cols = static_cast<float>(b.cols);
    x = b.rms ? 0.0f : sum_group(x, sums) / cols;
    y = sum_group(y, sums) / cols;
  }
  const float pr = b.post_weight ? a.post_rstd[row] : 1.0f;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kBlock * 8) {
    const int64_t left = b.cols - c;
    backward_values<T>(a, row, c, along, across, t);
    load_parameter<T>(b.post_weight, f32, c, left, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (b.post_weight) t.df[e] = pr * (t.df[e] * w[e] - x - t.post[e] * y);
      t.f[e] *= t.g[e];
      t.g[e] *= b.scale;
    }
    if (a.dx) store8_upto(static_cast<T*>(a.dx) + row * a.lddx + c, left, t.g);
    if (a.dh) store8_upto(static_cast<T*>(a.dh) + row * a.lddh + c, left, t.df);
    if (a.dgate) store8_upto(static_cast<T*>(a.dgate) + row * a.lddgate + c, left, t.f);
  }
}

// partial[chunk][5][cols]
constexpr int kSums = 5;
template <typename T>
__global__ __launch_bounds__(64) void k_residual_dw(ResidualNormBackward a, Chunks chunks,
                                                    const float2* means, float* partial) {
  const int chunk = blockIdx.y;
  int worker = 0;
  while (chunks.chunk0[worker + 1] <= chunk) ++worker;
  const int64_t begin = chunks.token0[worker] + (chunk - chunks.chunk0[worker]) * chunks.rows;
  const int64_t last = chunks.token0[worker + 1];
  const int64_t end = begin + chunks.rows < last ? begin + chunks.rows : last;
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x) * 8;
  if (c >= a.b.cols) return;
  float sum[kSums][8] = {};
  Eight t;
  for (int64_t row = begin; row < end; ++row) {
    const float2 m = means[row];
    backward_values<T>(a, row, c, m.x, m.y, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      sum[0][e] = __builtin_fmaf(t.dy[e], t.hat[e], sum[0][e]);
      sum[1][e] += t.dy[e];
      sum[2][e] = __builtin_fmaf(t.df[e], t.post[e], sum[2][e]);
      sum[3][e] += t.df[e];
      sum[4][e] = __builtin_fmaf(t.g[e], t.f[e], sum[4][e]);
    }
  }
  for (int k = 0; k < kSums; ++k)
    store8_upto(partial + (static_cast<int64_t>(chunk) * kSums + k) * a.b.cols + c, a.b.cols - c,
                sum[k]);
}

__global__ __launch_bounds__(kBlock) void k_residual_sums(const float* __restrict__ partial,
                                                          int64_t cols, Chunks chunks,
                                                          garfield_residual_gradients to) {
  const int k = blockIdx.y % kSums, worker = blockIdx.y / kSums;
  float* const outs[kSums] = {to.weight, to.bias, to.post_weight, to.post_bias, to.gate};
  const int64_t lds[kSums] = {to.ld_weight, to.ld_bias, to.ld_post_weight, to.ld_post_bias, to.ld_gate};
  if (!outs[k]) return;
  for (int64_t c = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; c < cols;
       c += static_cast<int64_t>(gridDim.x) * kBlock) {
    float sum = 0.0f;
    for (int i = chunks.chunk0[worker]; i < chunks.chunk0[worker + 1]; ++i)
      sum += partial[(static_cast<int64_t>(i) * kSums + k) * cols + c];
    outs[k][worker * lds[k] + c] = sum;
  }
}

template <typename T>
void launch_backward(const ResidualNormBackward& a, const Chunks& c, void* workspace, hipStream_t s) {
  float2* means = static_cast<float2*>(workspace);
  float* partial = reinterpret_cast<float*>(means + a.b.rows);
  const garfield_residual_gradients& to = a.to;
  const bool sums = to.weight || to.bias || to.post_weight || to.post_bias || to.gate;
  if (a.b.rows > 0) {
    launch("residual_dx", k_residual_dx<T>, dim3(static_cast<uint32_t>(a.b.rows)), dim3(kBlock), 0,
           s, a, means);
    if (sums)
      launch("residual_dw", k_residual_dw<T>,
             dim3(static_cast<uint32_t>((a.b.cols + 511) / 512), c.chunk0[c.n]), dim3(64), 0, s, a,
             c, means, partial);
  }
  if (sums) {
    const int64_t groups = (a.b.cols + kBlock - 1) / kBlock, most = int64_t{1} << 15;
    launch("residual_sums", k_residual_sums,
           dim3(static_cast<uint32_t>(groups < most ? groups : most), c.n * kSums), dim3(kBlock), 0,
           s, partial, a.b.cols, c, to);
  }
}

}  // namespace

hipError_t enqueue_residual_norm(const ResidualNorm& a, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(a.b.rows));
  if (a.b.type == GARFIELD_F32) launch("residual_norm", k_residual_norm<float>, grid, dim3(kBlock), 0, s, a);
  else if (a.b.type == GARFIELD_BF16) launch("residual_norm", k_residual_norm<__bf16>, grid, dim3(kBlock), 0, s, a);
  else launch("residual_norm", k_residual_norm<_Float16>, grid, dim3(kBlock), 0, s, a);
  return hipGetLastError();
}

Chunks residual_norm_backward_chunks(const garfield_residual_block& b, int n,
                                     const int64_t* counts) {
  return make_chunks(n, counts, b.rows < 65536 ? 64 : b.rows / 1024);
}

size_t residual_norm_backward_bytes(const garfield_residual_block& b, const Chunks& c) {
  return b.rows * sizeof(float2) + static_cast<size_t>(c.chunk0[c.n]) * kSums * b.cols * sizeof(float);
}

hipError_t enqueue_residual_norm_backward(const ResidualNormBackward& a, const Chunks& c,
                                          void* workspace, hipStream_t s) {
  if (a.b.type == GARFIELD_F32) launch_backward<float>(a, c, workspace, s);
  else if (a.b.type == GARFIELD_BF16) launch_backward<__bf16>(a, c, workspace, s);
  else launch_backward<_Float16>(a, c, workspace, s);
  return hipGetLastError();
}

}  // namespace garfield
