// Layer norm of rows and its backward pass, with the weight's gradient of each
// worker.
//
// Both read a row once and keep it in registers: the mean, then the variance
// from the differences to it, then the outputs. Sums are fp32, the mean's across lanes
// fp64. A lane holds eight neighbouring columns at a time, so the 16 lanes of a DPP row
// hold one 8-bit block and its largest magnitude needs no memory. Long inputs are bound
// by memory (a copy runs at 4.7 TB/s, read and written), short ones by latency.

#include "block8.h"
#include "internal.h"
#include "row_sums.h"
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

// A row of 4096 columns in bf16 takes 3.2 us, 65536 of them with x8 280 us (4.8 TB/s).
// Rows of up to 512 * WAVES * NV columns, R rows at a time to a team of WAVES waves,
// NV vectors of eight of each to a lane. Workgroups of four waves hold 4 / WAVES
// teams. Several rows at a time share what is read of weight and bias, which is
// more bytes (from the caches) than the row itself.
template <typename T, int WAVES, int NV, int R>
__global__ __launch_bounds__(64 * (WAVES > 4 ? WAVES : 4)) void k_layernorm(LayerNorm a) {
  constexpr int kThreads = 64 * WAVES;
  constexpr int kTeams = WAVES > 4 ? 1 : 4 / WAVES;
  static_assert(WAVES == 1 || kTeams == 1, "barriers are the whole workgroup's");
  __shared__ double totals[WAVES][R];
  __shared__ float sums[WAVES][R];
  const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * kTeams + threadIdx.x / kThreads) * R;
  if (row0 >= a.rows) return;  // whole waves, and no barrier where there are several teams
  const int lane = threadIdx.x % kThreads, cols = static_cast<int>(a.cols);
  typename Pack8<T>::type x[R][NV];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = row0 + r < a.rows ? row0 + r : a.rows - 1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * kThreads + lane) * 8;
      x[r][j] = raw8_upto(static_cast<const T*>(a.x) + row * a.ldx + c, a.cols - c);
    }
  }
  float mean[R], rstd[R], v[8];
  double total[R];
  const float scale = static_cast<float>(a.share);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float sum = 0.0f, first = 0.0f;
    int count = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = cols - (j * kThreads + lane) * 8;
      unpack8<T>(x[r][j], v);
      if (j == 0) first = first_value(v[0]);
      if (left >= 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += v[e] - first;
        count += 8;
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += e < left ? v[e] - first : 0.0f;
        count += left > 0 ? left : 0;
      }
    }
    total[r] = lane_total(first, count, sum);
  }
  sums_group<WAVES, R>(total, totals);
#pragma unroll
  for (int r = 0; r < R; ++r) mean[r] = static_cast<float>(total[r] * a.share);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float square = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = cols - (j * kThreads + lane) * 8;
      unpack8<T>(x[r][j], v);
      if (left >= 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) square = __builtin_fmaf(v[e] - mean[r], v[e] - mean[r], square);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e < left) square = __builtin_fmaf(v[e] - mean[r], v[e] - mean[r], square);
      }
    }
    rstd[r] = square;
  }
  sums_group<WAVES, R>(rstd, sums);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    rstd[r] = 1.0f / __builtin_sqrtf(rstd[r] * scale + a.eps);
    if (lane == 0 && row0 + r < a.rows) {
      a.mean[row0 + r] = mean[r];
      a.rstd[row0 + r] = rstd[r];
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8, left = a.cols - c;
    float w[8], b[8] = {};
    if (a.y || a.y8.values) {
      load_weight<T>(a.weight, a.weight_f32, c, left, w);
      if (a.bias) load_weight<T>(a.bias, a.weight_f32, c, left, b);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = row0 + r;
      if (row >= a.rows) break;
      unpack8<T>(x[r][j], v);
      if (a.x8.values) store_blocks(a.x8, row, c, v);
      if (!a.y && !a.y8.values) continue;
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf((v[e] - mean[r]) * rstd[r], w[e], b[e]);
      if (left < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = e < left ? v[e] : 0.0f;
      }
      if (a.y) store8_upto(static_cast<T*>(a.y) + row * a.ldy + c, left, v);
      if (a.y8.values) store_blocks(a.y8, row, c, v);
    }
  }
}

// Longer rows: the workgroup reads its row three times.
template <typename T>
__global__ __launch_bounds__(1024) void k_layernorm_long(LayerNorm a) {
  constexpr int kThreads = 1024;
  __shared__ double totals[16];
  __shared__ float sums[16];
  const int64_t row = blockIdx.x;
  const T* x = static_cast<const T*>(a.x) + row * a.ldx;
  const int64_t padded = (a.cols + 511) / 512 * 512;  // four blocks
  float v[8];
  const int64_t c0 = threadIdx.x * 8;
  const float first = c0 < a.cols ? first_value(static_cast<float>(x[c0])) : 0.0f;
  double total = 0.0;
  for (int64_t c = c0; c < a.cols; c += kThreads * 8) {
    load8_upto(x + c, a.cols - c, v);
    float sum = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) sum += c + e < a.cols ? v[e] - first : 0.0f;
    total += lane_total(first, a.cols - c < 8 ? static_cast<int>(a.cols - c) : 8, sum);
  }
  const float mean = static_cast<float>(sum_group<16>(total, totals) * a.share);
  float square = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < a.cols; c += kThreads * 8) {
    load8_upto(x + c, a.cols - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = c + e < a.cols ? v[e] - mean : 0.0f;
      square = __builtin_fmaf(t, t, square);
    }
  }
  const float var = sum_group<16>(square, sums) / static_cast<float>(a.cols);
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

template <typename T, int WAVES, int NV, int R>
void launch_layernorm(const LayerNorm& a, hipStream_t s) {
  constexpr int kRows = WAVES > 4 ? R : 4 / WAVES * R;
  launch("layernorm", k_layernorm<T, WAVES, NV, R>,
         dim3(static_cast<uint32_t>((a.rows + kRows - 1) / kRows)),
         dim3(64 * (WAVES > 4 ? WAVES : 4)), 0, s, a);
}

// With many rows two at a time share the reads of weight and bias and the barriers:
// 65536 x 4096 in bf16 takes 200 us (5.4 TB/s, a copy's rate), one at a time 235; 32768 x 2048
// with y8 67, one at a time 76. (With plain fp32 sums in the mean, 212 us: four rows at a
// time 218, a wave to a row of its own 211, but 74 against 67 at 32768 x 2048 with y8.)
template <typename T>
void choose_layernorm(const LayerNorm& a, hipStream_t s) {
  const bool many = a.rows >= 8 * device_cus();
  if (a.cols > 32768)
    launch("layernorm_long", k_layernorm_long<T>, dim3(static_cast<uint32_t>(a.rows)), dim3(1024),
           0, s, a);
  else if (a.cols > 16384) launch_layernorm<T, 16, 4, 1>(a, s);
  else if (a.cols > 8192) launch_layernorm<T, 16, 2, 1>(a, s);
  else if (a.cols > 4096) launch_layernorm<T, 4, 4, 1>(a, s);
  else if (many && a.cols > 2048) launch_layernorm<T, 4, 2, 2>(a, s);
  else if (many && a.cols > 1024) launch_layernorm<T, 4, 1, 2>(a, s);
  else if (a.cols > 2048) launch_layernorm<T, 4, 2, 1>(a, s);
  else if (a.cols > 1024) launch_layernorm<T, 4, 1, 1>(a, s);
  else if (a.cols > 512) launch_layernorm<T, 1, 2, 1>(a, s);
  else launch_layernorm<T, 1, 1, 1>(a, s);
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

// A workgroup goes through one chunk of a worker's rows (up to 8 * THREADS * NV
// columns), its share of the weight's gradient in registers, and writes that to
// partial[chunk][2][cols]; k_sum_chunks adds the chunks of a worker. R rows are worked
// on at a time, with one barrier for their sums, while the next R are on their way.
// 32768 x 4096 of 19 workers in bf16, x in 8 bits: 144 us, 4.7 TB/s (one row at a time
// without the next on its way: 245), and 7 us for the sums.
template <typename T, bool X8, int THREADS, int NV, int R>
__global__ __launch_bounds__(THREADS) void k_layernorm_backward(LayerNormBackward a, Chunks chunks,
                                                                float* partial) {
  constexpr int kWaves = THREADS / 64;
  typedef typename Pack8<T>::type Raw;
  __shared__ float sums[2][kWaves][2 * R];
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
  // a row as it lies in memory: dy, and x or its codes and exponents
  Raw dy[R][NV], x[X8 ? 1 : R][NV];
  u2 code[X8 ? R : 1][NV];
  int shift[X8 ? R : 1][NV];
  float mean[R], rstd[R];
  auto fetch = [&](int64_t row0) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = row0 + r < end ? row0 + r : end - 1;
      mean[r] = a.mean[row];
      rstd[r] = a.rstd[row];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int64_t c = (j * THREADS + threadIdx.x) * 8;
        dy[r][j] = raw8_upto(static_cast<const T*>(a.dy) + row * a.lddy + c, a.cols - c);
        if constexpr (X8) {
          const int64_t at = c < a.cols ? c : 0;
          code[r][j] = *reinterpret_cast<const u2*>(a.x8.values + row * a.x8.ld_values + at);
          shift[r][j] = a.x8.exponents[row * a.x8.ld_exponents + at / kBlock8];
        } else {
          x[r][j] = raw8_upto(static_cast<const T*>(a.x) + row * a.ldx + c, a.cols - c);
        }
      }
    }
  };
  fetch(begin);
  for (int64_t row0 = begin; row0 < end; row0 += R) {
    float g[R][NV][8], h[R][NV][8], m[R], d[R], both[2 * R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      m[r] = mean[r];
      d[r] = rstd[r];
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        unpack8<T>(dy[r][j], g[r][j]);
        if constexpr (X8) decode8(code[r][j], power2(shift[r][j] - 127), h[r][j]);
        else unpack8<T>(x[r][j], h[r][j]);
      }
    }
    if (row0 + R < end) fetch(row0 + R);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float along = 0.0f, across = 0.0f;
      if (r == 0 || row0 + r < end) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
          for (int e = 0; e < 8; ++e) h[r][j][e] = (h[r][j][e] - m[r]) * d[r];
          const int64_t left = a.cols - (j * THREADS + threadIdx.x) * 8;
          if (left < 8) {
#pragma unroll
            for (int e = 0; e < 8; ++e) h[r][j][e] = e < left ? h[r][j][e] : 0.0f;
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            dw[j][e] = __builtin_fmaf(g[r][j][e], h[r][j][e], dw[j][e]);
            db[j][e] += g[r][j][e];
            g[r][j][e] *= w[j][e];
            along += g[r][j][e];
            across = __builtin_fmaf(g[r][j][e], h[r][j][e], across);
          }
        }
      }
      both[2 * r] = along;
      both[2 * r + 1] = across;
    }
    if (!a.dx) continue;
    // the sums alternate between two places: one barrier for R rows
    sums_group<kWaves, 2 * R>(both, sums[(row0 - begin) / R & 1]);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (r > 0 && row0 + r >= end) break;
      const float along = both[2 * r] * scale, across = both[2 * r + 1] * scale;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int64_t c = (j * THREADS + threadIdx.x) * 8;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          g[r][j][e] = d[r] * (g[r][j][e] - along - h[r][j][e] * across);
        if (c < a.cols)
          store8_upto(static_cast<T*>(a.dx) + (row0 + r) * a.lddx + c, a.cols - c, g[r][j]);
      }
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

// Longer rows: dx from two reads of the row, the weight's gradient by columns, a third.
// 8192 x 16384 of 19 workers in bf16, x in 8 bits: 188 us for dx, 87 for the chunks' sums and 13
// for the workers', 2.3 TB/s of what a single read would take.
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

// The chunks of a worker added in one order: 64 columns of partial[chunk][2][cols] at a
// time for worker blockIdx.y, every fourth chunk to a wave.
__global__ __launch_bounds__(kBlock) void k_sum_chunks(const float* __restrict__ partial,
                                                       int64_t cols, Chunks chunks,
                                                       float* __restrict__ dweight,
                                                       int64_t ld_dweight,
                                                       float* __restrict__ dbias,
                                                       int64_t ld_dbias) {
  __shared__ float sums[4][64];
  const int lane = threadIdx.x % 64, part = threadIdx.x / 64, worker = blockIdx.y;
  for (int64_t i0 = static_cast<int64_t>(blockIdx.x) * 64; i0 < 2 * cols;
       i0 += static_cast<int64_t>(gridDim.x) * 64) {
    const int64_t i = i0 + lane;
    float sum = 0.0f;
    if (i < 2 * cols) {
#pragma unroll 8
      for (int c = chunks.chunk0[worker] + part; c < chunks.chunk0[worker + 1]; c += 4)
        sum += partial[static_cast<int64_t>(c) * 2 * cols + i];
    }
    sums[part][lane] = sum;
    __syncthreads();
    if (part == 0 && i < 2 * cols) {
      sum = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
      if (i < cols) {
        if (dweight) dweight[worker * ld_dweight + i] = sum;
      } else if (dbias) {
        dbias[worker * ld_dbias + i - cols] = sum;
      }
    }
    __syncthreads();  // the sums' places are free
  }
}

template <typename T, bool X8, int THREADS, int NV, int R>
void launch_backward(const LayerNormBackward& a, const Chunks& c, float* partial, hipStream_t s) {
  launch("layernorm_backward", k_layernorm_backward<T, X8, THREADS, NV, R>, dim3(c.chunk0[c.n]),
         dim3(THREADS), 0, s, a, c, partial);
}

constexpr int64_t kBackwardMaxCols = 8192;

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
  } else if (a.cols > 4096) {
    launch_backward<T, X8, 512, 2, 1>(a, c, partial, s);
  } else if (a.cols > 2048) {
    launch_backward<T, X8, 512, 1, 2>(a, c, partial, s);
  } else if (a.cols > 1024) {
    launch_backward<T, X8, 256, 1, 2>(a, c, partial, s);
  } else if (a.cols > 512) {
    launch_backward<T, X8, 128, 1, 2>(a, c, partial, s);
  } else {
    launch_backward<T, X8, 64, 1, 2>(a, c, partial, s);
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

// Chunks of equal length, as many as the workgroups that the card holds at once (by
// their registers: 256, 512, 1024, 2048 or 4096 on 256 CUs) and no more: twelve more
// than 512 cost as much as 512.
Chunks layernorm_backward_chunks(int64_t rows, int64_t cols, int n, const int64_t* counts) {
  const int per_cu = cols > 4096 ? 1 : cols > 2048 ? 2 : cols > 1024 ? 4 : cols > 512 ? 8 : 16;
  const int64_t want = static_cast<int64_t>(device_cus()) * per_cu;
  int64_t per = (rows + want - 1) / want;
  per = per < 2 ? 2 : per;  // the rows that are worked on at a time
  Chunks c = make_chunks(n, counts, per);
  while (c.chunk0[n] > want && per < rows) {
    per += (per + 31) / 32;
    c = make_chunks(n, counts, per);
  }
  return c;
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
  if (a.dweight || a.dbias) {
    // a workgroup for 64 columns, up to 2^23 of them: a launch has fewer than 2^32 threads
    const int64_t groups = (2 * a.cols + 63) / 64, most = int64_t{1} << 23;
    launch("sum_chunks", k_sum_chunks,
           dim3(static_cast<uint32_t>(groups < most ? groups : most), c.n), dim3(kBlock), 0, s,
           partial, a.cols, c, a.dweight, a.ld_dweight, a.dbias, a.ld_dbias);
  }
  return hipGetLastError();
}

}  // namespace garfield
