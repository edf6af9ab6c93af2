// Layer norm of rows and its backward pass, with the weight's gradient of each
// worker.
//
// Both read a row once and keep it in registers: the mean, then the variance
// from the differences to it, then the outputs. All sums are fp32. A lane holds
// eight neighbouring columns at a time, so the 16 lanes of a DPP row hold one
// 8-bit block and its largest magnitude needs no memory.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

Chunks make_chunks(int n, const int64_t* counts, int64_t rows) {
  Chunks c;
  c.n = n;
  c.rows = rows;
  for (int w = 0; w < n; ++w) {
    c.token0[w + 1] = c.token0[w] + counts[w];
    c.chunk0[w + 1] = c.chunk0[w] + static_cast<int>((counts[w] + rows - 1) / rows);
  }
  return c;
}

namespace {

// Sum over the workgroup of `waves` waves; the same value in every thread.
// `at` holds one float a wave and is free again after the next barrier.
template <int WAVES>
__device__ __forceinline__ float sum_group(float v, float* at) {
  v = sum_wave(v);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += at[w];
  }
  return v;
}

// Weights of wtype at p[c..c+7] (cols beyond `left` read as 0).
template <typename T>
__device__ __forceinline__ void load_weight(const void* p, bool f32, int64_t c, int64_t left,
                                            float* v) {
  if (f32) load8_upto(static_cast<const float*>(p) + c, left, v);
  else load8_upto(static_cast<const T*>(p) + c, left, v);
}

// Eight values (0 beyond the row's end) of a row's columns c..c+7 as blocks.
// Called by all 16 lanes of a block.
__device__ __forceinline__ void store_blocks(const garfield_block8& out, int64_t row, int64_t c,
                                             const float* v) {
  float a = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = __builtin_fmaxf(a, magnitude(v[e]));
  const int s = block_shift(max16(a));
  const int64_t blocks = (out.cols + kBlock8 - 1) / kBlock8;
  const int64_t b = c / kBlock8;
  if (b < blocks)
    *reinterpret_cast<u2*>(out.values + row * out.ld_values + c) = encode8(v, s);
  if (c % kBlock8 == 0 && b < (blocks + 3) / 4 * 4)
    out.exponents[row * out.ld_exponents + b] = static_cast<uint8_t>(b < blocks ? s + 127 : 127);
}

// Rows of up to 512 * WAVES * NV columns: a row to WAVES waves, NV vectors of
// eight to a lane. Workgroups of four waves hold 4 / WAVES rows.
template <typename T, int WAVES, int NV>
__global__ __launch_bounds__(64 * (WAVES > 4 ? WAVES : 4)) void k_layernorm(LayerNorm a) {
  constexpr int kThreads = 64 * WAVES;
  constexpr int kRows = WAVES > 4 ? 1 : 4 / WAVES;
  static_assert(WAVES == 1 || kRows == 1, "barriers are the whole workgroup's");
  __shared__ float sums[2][WAVES];
  const int64_t row = static_cast<int64_t>(blockIdx.x) * kRows + threadIdx.x / kThreads;
  if (row >= a.rows) return;  // whole waves, and no barrier where kRows > 1
  const int lane = threadIdx.x % kThreads;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  float v[NV][8];
  float sum = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8;
    load8_upto(x + c, a.cols - c, v[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[j][e];
  }
  const float mean = sum_group<WAVES>(sum, sums[0]) / static_cast<float>(a.cols);
  float square = 0.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = c + e < a.cols ? v[j][e] - mean : 0.0f;
      square = __builtin_fmaf(t, t, square);
    }
  }
  const float var = sum_group<WAVES>(square, sums[1]) / static_cast<float>(a.cols);
  const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
  if (lane == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8;
    if (a.x8.values) store_blocks(a.x8, row, c, v[j]);
    if (!a.y && !a.y8.values) continue;
    float w[8], b[8] = {};
    load_weight<T>(a.weight, a.weight_f32, c, a.cols - c, w);
    if (a.bias) load_weight<T>(a.bias, a.weight_f32, c, a.cols - c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[j][e] = c + e < a.cols ? __builtin_fmaf((v[j][e] - mean) * rstd, w[e], b[e]) : 0.0f;
    if (a.y) store8_upto(static_cast<T*>(a.y) + row * a.ldy + c, a.cols - c, v[j]);
    if (a.y8.values) store_blocks(a.y8, row, c, v[j]);
  }
}

// Longer rows: the workgroup reads its row three times.
template <typename T>
__global__ __launch_bounds__(1024) void k_layernorm_long(LayerNorm a) {
  constexpr int kThreads = 1024;
  __shared__ float sums[2][16];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const int64_t padded = (a.cols + 511) / 512 * 512;  // four blocks
  float v[8];
  float sum = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
    load8_upto(x + c, a.cols - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += v[e];
  }
  const float mean = sum_group<16>(sum, sums[0]) / static_cast<float>(a.cols);
  float square = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
    load8_upto(x + c, a.cols - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = c + e < a.cols ? v[e] - mean : 0.0f;
      square = __builtin_fmaf(t, t, square);
    }
  }
  const float var = sum_group<16>(square, sums[1]) / static_cast<float>(a.cols);
  const float rstd = 1.0f / __builtin_sqrtf(var + a.eps);
  if (threadIdx.x == 0) {
    a.mean[row] = mean;
    a.rstd[row] = rstd;
  }
  for (int64_t c = threadIdx.x * 8; c < padded; c += kThreads * 8) {
    load8_upto(x + c, a.cols - c, v);
    if (a.x8.values) store_blocks(a.x8, row, c, v);
    if (!a.y && !a.y8.values) continue;
    float w[8], b[8] = {};
    load_weight<T>(a.weight, a.weight_f32, c, a.cols - c, w);
    if (a.bias) load_weight<T>(a.bias, a.weight_f32, c, a.cols - c, b);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = c + e < a.cols ? __builtin_fmaf((v[e] - mean) * rstd, w[e], b[e]) : 0.0f;
    if (a.y) store8_upto(static_cast<T*>(a.y) + row * a.ldy + c, a.cols - c, v);
    if (a.y8.values) store_blocks(a.y8, row, c, v);
  }
}

template <typename T, int WAVES, int NV>
void launch_layernorm(const LayerNorm& a, hipStream_t s) {
  constexpr int kRows = WAVES > 4 ? 1 : 4 / WAVES;
  launch("layernorm", k_layernorm<T, WAVES, NV>,
         dim3(static_cast<uint32_t>((a.rows + kRows - 1) / kRows)),
         dim3(64 * (WAVES > 4 ? WAVES : 4)), 0, s, a);
}

template <typename T>
void choose_layernorm(const LayerNorm& a, hipStream_t s) {
  if (a.cols > 65536)
    launch("layernorm_long", k_layernorm_long<T>, dim3(static_cast<uint32_t>(a.rows)), dim3(1024),
           0, s, a);
  else if (a.cols > 32768) launch_layernorm<T, 16, 8>(a, s);
  else if (a.cols > 16384) launch_layernorm<T, 16, 4>(a, s);
  else if (a.cols > 8192) launch_layernorm<T, 16, 2>(a, s);
  else if (a.cols > 4096) launch_layernorm<T, 4, 4>(a, s);
  else if (a.cols > 2048) launch_layernorm<T, 4, 2>(a, s);
  else if (a.cols > 1024) launch_layernorm<T, 1, 4>(a, s);
  else if (a.cols > 512) launch_layernorm<T, 1, 2>(a, s);
  else launch_layernorm<T, 1, 1>(a, s);
}

// ---------------------------------------------------------------------------
// Eight columns of a row of x, from the matrix or from its checkpoint.
template <typename T, bool X8>
__device__ __forceinline__ void load_x(const LayerNormBackward& a, int64_t row, int64_t c,
                                       float* v) {
  if constexpr (X8) {
    if (c < a.cols) {  // the padding holds zeros
      const int s = a.x8.exponents[row * a.x8.ld_exponents + c / kBlock8] - 127;
      decode8(*reinterpret_cast<const u2*>(a.x8.values + row * a.x8.ld_values + c), power2(s), v);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = 0.0f;
    }
  } else {
    load8_upto(static_cast<const T*>(a.x) + row * a.ldx + c, a.cols - c, v);
  }
}

// The worker whose chunk it is: as many workers end at or before it.
__device__ __forceinline__ int worker_of(const Chunks& c, int chunk) {
  const int lane = threadIdx.x % 64;
  static_assert(kWorkersMax == 64, "a lane looks at one worker");
  return __builtin_popcountll(__ballot(lane < c.n && c.chunk0[lane + 1] <= chunk));
}

// A workgroup goes through one chunk of a worker's rows (up to 8 * THREADS * NV
// columns), its share of the weight's gradient in registers, and writes that to
// partial[chunk][2][cols]; k_sum_chunks adds the chunks of a worker.
template <typename T, bool X8, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void k_layernorm_backward(LayerNormBackward a, Chunks chunks,
                                                                float* partial) {
  constexpr int kWaves = THREADS / 64;
  __shared__ float sums[2][2][kWaves];
  const int chunk = blockIdx.x;
  const int worker = worker_of(chunks, chunk);
  const int64_t begin = chunks.token0[worker] + (chunk - chunks.chunk0[worker]) * chunks.rows;
  const int64_t last = chunks.token0[worker + 1];
  const int64_t end = begin + chunks.rows < last ? begin + chunks.rows : last;
  const float scale = 1.0f / static_cast<float>(a.cols);
  float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * THREADS + threadIdx.x) * 8;
    load_weight<T>(a.weight, a.weight_f32, c, a.cols - c, w[j]);
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[j][e] = db[j][e] = 0.0f;
  }
  for (int64_t row = begin; row < end; ++row) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    float g[NV][8], h[NV][8];
    float along = 0.0f, across = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8;
      load8_upto(static_cast<const T*>(a.dy) + row * a.lddy + c, a.cols - c, g[j]);
      load_x<T, X8>(a, row, c, h[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        h[j][e] = (h[j][e] - mean) * rstd;
        dw[j][e] = __builtin_fmaf(g[j][e], h[j][e], dw[j][e]);
        db[j][e] += g[j][e];
        g[j][e] *= w[j][e];
        along += c + e < a.cols ? g[j][e] : 0.0f;
        across = c + e < a.cols ? __builtin_fmaf(g[j][e], h[j][e], across) : across;
      }
    }
    if (!a.dx) continue;
    // the rows' sums alternate between two places: one barrier a row
    float* at = sums[(row - begin) & 1][0];
    along = sum_wave(along);
    across = sum_wave(across);
    if constexpr (kWaves > 1) {
      if (threadIdx.x % 64 == 0) {
        at[threadIdx.x / 64] = along;
        at[kWaves + threadIdx.x / 64] = across;
      }
      __syncthreads();
      along = across = 0.0f;
#pragma unroll
      for (int i = 0; i < kWaves; ++i) {
        along += at[i];
        across += at[kWaves + i];
      }
    }
    along *= scale;
    across *= scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) g[j][e] = rstd * (g[j][e] - along - h[j][e] * across);
      if (c < a.cols)
        store8_upto(static_cast<T*>(a.dx) + row * a.lddx + c, a.cols - c, g[j]);
    }
  }
  float* out = partial + static_cast<int64_t>(chunk) * 2 * a.cols;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * THREADS + threadIdx.x) * 8;
    if (c >= a.cols) break;
    store8_upto(out + c, a.cols - c, dw[j]);
    store8_upto(out + a.cols + c, a.cols - c, db[j]);
  }
}

// Longer rows: dx from two reads of the row, the weight's gradient by columns.
template <typename T, bool X8>
__global__ __launch_bounds__(1024) void k_layernorm_dx_long(LayerNormBackward a) {
  constexpr int kThreads = 1024;
  __shared__ float sums[2][16];
  const int64_t row = blockIdx.x;
  const float mean = a.mean[row], rstd = a.rstd[row];
  const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
  float along = 0.0f, across = 0.0f;
  float g[8], h[8], w[8];
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
    load8_upto(dy + c, a.cols - c, g);
    load_x<T, X8>(a, row, c, h);
    load_weight<T>(a.weight, a.weight_f32, c, a.cols - c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= a.cols) continue;
      along = __builtin_fmaf(g[e], w[e], along);
      across = __builtin_fmaf(g[e] * w[e], (h[e] - mean) * rstd, across);
    }
  }
  along = sum_group<16>(along, sums[0]) / static_cast<float>(a.cols);
  across = sum_group<16>(across, sums[1]) / static_cast<float>(a.cols);
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
    load8_upto(dy + c, a.cols - c, g);
    load_x<T, X8>(a, row, c, h);
    load_weight<T>(a.weight, a.weight_f32, c, a.cols - c, w);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      g[e] = rstd * (g[e] * w[e] - along - (h[e] - mean) * rstd * across);
    store8_upto(static_cast<T*>(a.dx) + row * a.lddx + c, a.cols - c, g);
  }
}

template <typename T, bool X8>
__global__ __launch_bounds__(64) void k_layernorm_dw_long(LayerNormBackward a, Chunks chunks,
                                                          float* partial) {
  const int chunk = blockIdx.y;
  const int worker = worker_of(chunks, chunk);
  const int64_t begin = chunks.token0[worker] + (chunk - chunks.chunk0[worker]) * chunks.rows;
  const int64_t last = chunks.token0[worker + 1];
  const int64_t end = begin + chunks.rows < last ? begin + chunks.rows : last;
  const int64_t c = (static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x) * 8;
  if (c >= a.cols) return;
  float dw[8] = {}, db[8] = {}, g[8], h[8];
  for (int64_t row = begin; row < end; ++row) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    load8_upto(static_cast<const T*>(a.dy) + row * a.lddy + c, a.cols - c, g);
    load_x<T, X8>(a, row, c, h);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      dw[e] = __builtin_fmaf(g[e], (h[e] - mean) * rstd, dw[e]);
      db[e] += g[e];
    }
  }
  float* out = partial + static_cast<int64_t>(chunk) * 2 * a.cols;
  store8_upto(out + c, a.cols - c, dw);
  store8_upto(out + a.cols + c, a.cols - c, db);
}

// The chunks of a worker added in ascending order: column blockIdx.x * 256 +
// threadIdx.x of partial[chunk][2][cols] for worker blockIdx.y.
__global__ __launch_bounds__(kBlock) void k_sum_chunks(const float* __restrict__ partial,
                                                       int64_t cols, Chunks chunks,
                                                       float* __restrict__ dweight,
                                                       int64_t ld_dweight,
                                                       float* __restrict__ dbias,
                                                       int64_t ld_dbias) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= 2 * cols) return;
  const int worker = blockIdx.y;
  float sum = 0.0f;
#pragma unroll 8
  for (int c = chunks.chunk0[worker]; c < chunks.chunk0[worker + 1]; ++c)
    sum += partial[static_cast<int64_t>(c) * 2 * cols + i];
  if (i < cols) {
    if (dweight) dweight[worker * ld_dweight + i] = sum;
  } else if (dbias) {
    dbias[worker * ld_dbias + i - cols] = sum;
  }
}

template <typename T, bool X8, int THREADS, int NV>
void launch_backward(const LayerNormBackward& a, const Chunks& c, float* partial, hipStream_t s) {
  launch("layernorm_backward", k_layernorm_backward<T, X8, THREADS, NV>, dim3(c.chunk0[c.n]),
         dim3(THREADS), 0, s, a, c, partial);
}

constexpr int64_t kBackwardMaxCols = 16384;

template <typename T, bool X8>
void choose_backward(const LayerNormBackward& a, const Chunks& c, float* partial, hipStream_t s) {
  if (a.cols > kBackwardMaxCols) {
    if (a.dx)
      launch("layernorm_dx_long", k_layernorm_dx_long<T, X8>, dim3(static_cast<uint32_t>(a.rows)),
             dim3(1024), 0, s, a);
    if (a.dweight || a.dbias)
      launch("layernorm_dw_long", k_layernorm_dw_long<T, X8>,
             dim3(static_cast<uint32_t>((a.cols + 511) / 512), c.chunk0[c.n]), dim3(64), 0, s, a,
             c, partial);
  } else if (a.cols > 8192) {
    launch_backward<T, X8, 1024, 2>(a, c, partial, s);
  } else if (a.cols > 4096) {
    launch_backward<T, X8, 512, 2>(a, c, partial, s);
  } else if (a.cols > 2048) {
    launch_backward<T, X8, 256, 2>(a, c, partial, s);
  } else if (a.cols > 1024) {
    launch_backward<T, X8, 256, 1>(a, c, partial, s);
  } else if (a.cols > 512) {
    launch_backward<T, X8, 128, 1>(a, c, partial, s);
  } else {
    launch_backward<T, X8, 64, 1>(a, c, partial, s);
  }
}

template <typename T>
void choose_x(const LayerNormBackward& a, const Chunks& c, float* partial, hipStream_t s) {
  if (a.x) choose_backward<T, false>(a, c, partial, s);
  else choose_backward<T, true>(a, c, partial, s);
}

}  // namespace

hipError_t enqueue_layernorm(const LayerNorm& a, int type, hipStream_t s) {
  if (type == GARFIELD_F32) choose_layernorm<float>(a, s);
  else if (type == GARFIELD_BF16) choose_layernorm<__bf16>(a, s);
  else choose_layernorm<_Float16>(a, s);
  return hipGetLastError();
}

// Chunks of equal length, so many that they fill the card: about two
// workgroups of four waves a CU.
Chunks layernorm_backward_chunks(int64_t rows, int64_t cols, int n, const int64_t* counts) {
  const int64_t want = cols > 2048 ? 512 : cols > 512 ? 1024 : 2048;
  const int64_t per = (rows + want - 1) / want;
  return make_chunks(n, counts, per < 1 ? 1 : per);
}

size_t layernorm_backward_bytes(const Chunks& c, int64_t cols) {
  return static_cast<size_t>(c.chunk0[c.n]) * 2 * cols * sizeof(float);
}

hipError_t enqueue_layernorm_backward(const LayerNormBackward& a, int type, const Chunks& c,
                                      void* workspace, hipStream_t s) {
  float* partial = static_cast<float*>(workspace);
  if (a.rows > 0) {
    if (type == GARFIELD_F32) choose_x<float>(a, c, partial, s);
    else if (type == GARFIELD_BF16) choose_x<__bf16>(a, c, partial, s);
    else choose_x<_Float16>(a, c, partial, s);
  }
  if (a.dweight || a.dbias)
    launch("sum_chunks", k_sum_chunks,
           dim3(static_cast<uint32_t>((2 * a.cols + kBlock - 1) / kBlock), c.n), dim3(kBlock), 0,
           s, partial, a.cols, c, a.dweight, a.ld_dweight, a.dbias, a.ld_dbias);
  return hipGetLastError();
}

}  // namespace garfield
