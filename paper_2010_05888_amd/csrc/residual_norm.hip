// The residual around a block with the norms before and after it, and its backward pass with
// the parameters' gradients of each worker.
//
// Bound by memory: both passes read every value once and keep a row in registers between the
// sums over it, one after the other: N_post's mean, its deviation, then N's (the stream is known
// only then); back, N's two sums and then N_post's. 65536 x 4096 in bf16 with y8 takes 510 us (4.75
// TB/s; a copy runs at 5.26), 19 workers' 32768 x 4096 back with a gate of tokens 431 (5.0).
// Means are kept as layer norm's are: differences to a lane's first value, fp64 across lanes.

#include "block8.h"
#include "internal.h"
#include "row_sums.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

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

constexpr int kLong = 1024, kLongWaves = kLong / 64;  // threads to a row that is read again and again

// Mean (0 with rms) and 1 / deviation of a row, `values` giving eight columns of it.
template <typename F>
__device__ __forceinline__ void long_statistics(const garfield_residual_block& b, double share,
                                           double* totals, float* sums, F&& values, float* mean,
                                           float* rstd) {
  float v[8];
  *mean = 0.0f;
  if (!b.rms) {
    double sum = 0.0;
    for (int64_t c = threadIdx.x * 8; c < b.cols; c += kLong * 8) {
      values(c, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += c + e < b.cols ? v[e] : 0.0f;
    }
    *mean = static_cast<float>(sum_group<kLongWaves>(sum, totals) * share);
  }
  float square = 0.0f;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kLong * 8) {
    values(c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float t = c + e < b.cols ? v[e] - *mean : 0.0f;
      square = __builtin_fmaf(t, t, square);
    }
  }
  square = sum_group<kLongWaves>(square, sums);
  *rstd = 1.0f / __builtin_sqrtf(square * static_cast<float>(share) + b.eps);
}

// Mean (0 with rms) and 1 / deviation of R rows that a team of WAVES waves holds, NV vectors of
// eight columns of each to a lane: values(r, j, v) gives them.
template <int WAVES, int NV, int R, typename F>
__device__ __forceinline__ void statistics(const garfield_residual_block& b, double share, int lane,
                                           double (*totals)[R], float (*sums)[R], F&& values,
                                           float* mean, float* rstd) {
  constexpr int kThreads = 64 * WAVES;
  const int cols = static_cast<int>(b.cols);
  float v[8];
  if (b.rms) {
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = 0.0f;
  } else {
    double total[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float sum = 0.0f, first = 0.0f;
      int count = 0;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int left = cols - (j * kThreads + lane) * 8;
        values(r, j, v);
        if (j == 0) first = first_value(v[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += left >= 8 || e < left ? v[e] - first : 0.0f;
        count += left >= 8 ? 8 : left > 0 ? left : 0;
      }
      total[r] = lane_total(first, count, sum);
    }
    sums_group<WAVES, R>(total, totals);
#pragma unroll
    for (int r = 0; r < R; ++r) mean[r] = static_cast<float>(total[r] * share);
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float square = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int left = cols - (j * kThreads + lane) * 8;
      values(r, j, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float t = left >= 8 || e < left ? v[e] - mean[r] : 0.0f;
        square = __builtin_fmaf(t, t, square);
      }
    }
    rstd[r] = square;
  }
  sums_group<WAVES, R>(rstd, sums);
  const float scale = static_cast<float>(share);
#pragma unroll
  for (int r = 0; r < R; ++r) rstd[r] = 1.0f / __builtin_sqrtf(rstd[r] * scale + b.eps);
}

// Rows of up to 512 * WAVES * NV columns, R rows at a time to a team of WAVES waves; workgroups
// of four waves hold 4 / WAVES teams. x and h are read once; the stream stays in registers in
// fp32 from its sum to its norm. Several rows at a time share the parameters' reads, which are
// more bytes (from the caches) than a row.
template <typename T, int WAVES, int NV, int R>
__global__ __launch_bounds__(64 * (WAVES > 4 ? WAVES : 4)) void k_residual_norm(ResidualNorm a) {
  constexpr int kThreads = 64 * WAVES;
  constexpr int kTeams = WAVES > 4 ? 1 : 4 / WAVES;
  static_assert(WAVES == 1 || kTeams == 1, "barriers are the whole workgroup's");
  __shared__ double totals[2][WAVES][R];
  __shared__ float sums[2][WAVES][R];
  const garfield_residual_block& b = a.b;
  const int64_t row0 = (static_cast<int64_t>(blockIdx.x) * kTeams + threadIdx.x / kThreads) * R;
  if (row0 >= b.rows) return;  // whole waves, and no barrier where there are several teams
  const int lane = threadIdx.x % kThreads;
  const bool f32 = b.wtype == GARFIELD_F32, by_tokens = b.gate && b.ld_gate;
  typedef typename Pack8<T>::type Raw;
  Raw x[R][NV], h[R][NV], gate[R][NV];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t row = row0 + r < b.rows ? row0 + r : b.rows - 1;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * kThreads + lane) * 8;
      h[r][j] = raw8_upto(static_cast<const T*>(a.h) + row * a.ldh + c, b.cols - c);
      x[r][j] = raw8_upto(static_cast<const T*>(a.x) + row * a.ldx + c, b.cols - c);
      if (by_tokens) gate[r][j] = raw8_upto(static_cast<const T*>(b.gate) + row * b.ld_gate + c, b.cols - c);
    }
  }
  float mean[R], rstd[R], s[R][NV][8];
  if (b.post_weight) {
    statistics<WAVES, NV, R>(b, a.share, lane, totals[0], sums[0],
                             [&](int r, int j, float* v) { unpack8<T>(h[r][j], v); }, mean, rstd);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (lane == 0 && row0 + r < b.rows) {
        if (!b.rms) a.post_mean[row0 + r] = mean[r];
        a.post_rstd[row0 + r] = rstd[r];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8, left = b.cols - c;
    float w[8], bias[8], g[8], t[8];
    if (b.post_weight) {
      load_weight<T>(b.post_weight, f32, c, left, w);
      load_parameter<T>(b.post_bias, f32, c, left, 0.0f, bias);
    }
    if (!by_tokens) load_parameter<T>(b.gate, f32, c, left, 1.0f, g);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float* v = s[r][j];
      unpack8<T>(h[r][j], v);
      unpack8<T>(x[r][j], t);
      if (b.post_weight) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = __builtin_fmaf((v[e] - mean[r]) * rstd[r], w[e], bias[e]);
      }
      if (by_tokens) unpack8<T>(gate[r][j], g);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = __builtin_fmaf(b.scale, t[e], g[e] * v[e]);
      if (row0 + r < b.rows)
        store8_upto(static_cast<T*>(a.s) + (row0 + r) * a.lds + c, left, v);
    }
  }
  if (!b.weight) return;
  statistics<WAVES, NV, R>(b, a.share, lane, totals[1], sums[1],
                           [&](int r, int j, float* v) {
#pragma unroll
                             for (int e = 0; e < 8; ++e) v[e] = s[r][j][e];
                           },
                           mean, rstd);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (lane == 0 && row0 + r < b.rows) {
      if (!b.rms) a.mean[row0 + r] = mean[r];
      a.rstd[row0 + r] = rstd[r];
    }
  }
  if (!a.y && !a.y8.values) return;
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int64_t c = (j * kThreads + lane) * 8, left = b.cols - c;
    float w[8], bias[8];
    load_weight<T>(b.weight, f32, c, left, w);
    load_parameter<T>(b.bias, f32, c, left, 0.0f, bias);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      const int64_t row = row0 + r;
      if (row >= b.rows) break;
      float* v = s[r][j];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = __builtin_fmaf((v[e] - mean[r]) * rstd[r], w[e], bias[e]);
        if (left < 8) v[e] = e < left ? v[e] : 0.0f;
      }
      if (a.y) store8_upto(static_cast<T*>(a.y) + row * a.ldy + c, left, v);
      if (a.y8.values) store_blocks(a.y8, row, c, v);
    }
  }
}

// Longer rows: the workgroup reads them again for each of its sums (4096 x 20000 in bf16 320 us,
// 2.0 TB/s of what one read would take).
template <typename T>
__global__ __launch_bounds__(kLong) void k_residual_norm_long(ResidualNorm a) {
  __shared__ double totals[2][kLongWaves];
  __shared__ float sums[2][kLongWaves];
  const int64_t row = blockIdx.x;
  float pm = 0.0f, pr = 1.0f, mean, rstd, v[8];
  if (a.b.post_weight) {
    long_statistics(a.b, a.share, totals[0], sums[0], [&](int64_t c, float* h) {
      load8_upto(static_cast<const T*>(a.h) + row * a.ldh + c, a.b.cols - c, h);
    }, &pm, &pr);
    if (threadIdx.x == 0) {
      if (!a.b.rms) a.post_mean[row] = pm;
      a.post_rstd[row] = pr;
    }
  }
  auto values = [&](int64_t c, float* t) { stream_values<T>(a, row, c, pm, pr, t); };
  if (a.b.weight) {
    long_statistics(a.b, a.share, totals[1], sums[1], values, &mean, &rstd);
    if (threadIdx.x == 0) {
      if (!a.b.rms) a.mean[row] = mean;
      a.rstd[row] = rstd;
    }
  }
  const bool f32 = a.b.wtype == GARFIELD_F32;
  const int64_t padded = (a.b.cols + 511) / 512 * 512;
  for (int64_t c = threadIdx.x * 8; c < padded; c += kLong * 8) {
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
    if (a.y8.values) store_blocks(a.y8, row, c, v);
  }
}

// ---------------------------------------------------------------------------
// Longer rows' backward pass: dx, dh and a gate of tokens from three reads of a row, then the
// parameters' gradients by columns, from a fourth: 8192 x 12288 in bf16 790 us, 1.5 TB/s of what
// one read would take. (Arrays indexed by a loop that is not unrolled live in scratch: 3100.)
// What it knows of eight columns of a row.
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
                                              float (*sums)[kLongWaves], float* along,
                                              float* across) {
  const garfield_residual_block& b = a.b;
  float x = 0.0f, y = 0.0f, w[8];
  Eight t;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kLong * 8) {
    backward_values<T>(a, row, c, 0.0f, 0.0f, t);
    load_parameter<T>(b.weight, b.wtype == GARFIELD_F32, c, b.cols - c, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (c + e >= b.cols) continue;
      x = __builtin_fmaf(t.dy[e], w[e], x);
      y = __builtin_fmaf(t.dy[e] * w[e], t.hat[e], y);
    }
  }
  const float cols = static_cast<float>(b.cols);
  x = sum_group<kLongWaves>(x, sums[0]) / cols;
  *along = b.rms ? 0.0f : x;
  *across = sum_group<kLongWaves>(y, sums[1]) / cols;
}

template <typename T>
__global__ __launch_bounds__(kLong) void k_residual_dx_long(ResidualNormBackward a, float2* means) {
  __shared__ float sums[4][kLongWaves];
  const garfield_residual_block& b = a.b;
  const int64_t row = blockIdx.x;
  float along = 0.0f, across = 0.0f, w[8];
  if (a.dy) backward_sums<T>(a, row, sums, &along, &across);
  if (threadIdx.x == 0) means[row] = {along, across};
  float x = 0.0f, y = 0.0f;
  Eight t;
  const bool f32 = b.wtype == GARFIELD_F32;
  if (b.post_weight) {
    for (int64_t c = threadIdx.x * 8; c < b.cols; c += kLong * 8) {
      backward_values<T>(a, row, c, along, across, t);
      load_parameter<T>(b.post_weight, f32, c, b.cols - c, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (c + e >= b.cols) continue;
        x = __builtin_fmaf(t.df[e], w[e], x);
        y = __builtin_fmaf(t.df[e] * w[e], t.post[e], y);
      }
    }
    const float cols = static_cast<float>(b.cols);
    x = sum_group<kLongWaves>(x, sums[2]) / cols;
    x = b.rms ? 0.0f : x;
    y = sum_group<kLongWaves>(y, sums[3]) / cols;
  }
  const float pr = b.post_weight ? a.post_rstd[row] : 1.0f;
  for (int64_t c = threadIdx.x * 8; c < b.cols; c += kLong * 8) {
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

// A worker's sums over its rows: weight, bias, post weight, post bias, gate; `sums` has a bit
// for each that is asked for, and partial[chunk][bit's rank][cols] a chunk's.
constexpr int kSums = 5;

// A workgroup goes through one chunk of a worker's rows (up to 8 * THREADS * NV columns), its
// share of the parameters' gradients in registers, and writes that to `partial`;
// k_residual_sums adds the chunks of a worker. One barrier for each norm's sums, while the next
// row is on its way. bf16 32768 x 4096 of 19 workers 290 us and 7 for the sums, 16384 x 8192 470 (all
// sums in registers, of which two thirds then are in scratch: 640).
// HOLD: the parameters and all sums stay in registers and the next row's ds and gate come early
// too; else the parameters are read again for every row, ds and the gate come under the first
// norm's sums, and all sums but the first live in LDS, each thread's own values.
template <typename T, int THREADS, int NV, bool HOLD>
__global__ __launch_bounds__(THREADS) void k_residual_backward(ResidualNormBackward a,
                                                               Chunks chunks, int sums_of,
                                                               float* partial) {
  constexpr int kWaves = THREADS / 64;
  typedef typename Pack8<T>::type Raw;
  __shared__ float sums[2][2][kWaves][2];
  constexpr int kHeld = HOLD ? kSums : 1;  // sums in registers
  __shared__ v4f totals[HOLD ? 1 : kSums - 1][NV][2][HOLD ? 1 : THREADS];
  const garfield_residual_block& b = a.b;
  const int chunk = blockIdx.x, worker = worker_of(chunks, chunk);
  const int64_t begin = chunks.token0[worker] + (chunk - chunks.chunk0[worker]) * chunks.rows;
  const int64_t last = chunks.token0[worker + 1];
  const int64_t end = begin + chunks.rows < last ? begin + chunks.rows : last;
  const float scale = 1.0f / static_cast<float>(b.cols);
  const bool f32 = b.wtype == GARFIELD_F32, by_tokens = b.gate && b.ld_gate;
  const bool post = b.post_weight != nullptr;
  float w[NV][8], pw[NV][8], pb[NV][8], gv[NV][8], total[kHeld][NV][8];
  auto parameter = [&](const void* p, float missing, float (&v)[NV][8]) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8;
      load_parameter<T>(p, f32, c, b.cols - c, missing, v[j]);
    }
  };
  const void* const columns = by_tokens ? nullptr : b.gate;
  if constexpr (HOLD) {
    parameter(b.weight, 0.0f, w);
    parameter(b.post_weight, 1.0f, pw);
    parameter(b.post_bias, 0.0f, pb);
    parameter(columns, 1.0f, gv);
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k)
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (k < kHeld) {
#pragma unroll
        for (int e = 0; e < 8; ++e) total[k < kHeld ? k : 0][j][e] = 0.0f;
      } else {
        totals[k - kHeld][j][0][threadIdx.x] = totals[k - kHeld][j][1][threadIdx.x] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
  // x * y (y null: x) of eight columns added to sum k
  auto add = [&](int k, int j, const float* x, const float* y) {
    if (k < kHeld) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float& t = total[k < kHeld ? k : 0][j][e];
        t = y ? __builtin_fmaf(x[e], y[e], t) : t + x[e];
      }
    } else {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        v4f t = totals[k - kHeld][j][half][threadIdx.x];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = half * 4 + e;
          t[e] = y ? __builtin_fmaf(x[i], y[i], t[e]) : t[e] + x[i];
        }
        totals[k - kHeld][j][half][threadIdx.x] = t;
      }
    }
  };
  Raw ds[NV], dy[NV], s[NV], h[NV], gate[NV];
  float mean = 0.0f, rstd = 1.0f, post_mean = 0.0f, post_rstd = 1.0f;
#pragma unroll
  for (int j = 0; j < NV; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) ds[j][e] = dy[j][e] = s[j][e] = static_cast<T>(0.0f);
  auto fetch = [&](int64_t row) {
    if (a.dy) {
      if (!b.rms) mean = a.mean[row];
      rstd = a.rstd[row];
    }
    if (post) {
      if (!b.rms) post_mean = a.post_mean[row];
      post_rstd = a.post_rstd[row];
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8, left = b.cols - c;
      auto of = [&](const void* p, int64_t ld) {
        return raw8_upto(static_cast<const T*>(p) + row * ld + c, left);
      };
      if (a.dy) {
        dy[j] = of(a.dy, a.lddy);
        s[j] = of(a.s, a.lds);
      }
      h[j] = of(a.h, a.ldh);
      if constexpr (HOLD) {
        if (a.ds) ds[j] = of(a.ds, a.ldds);
        if (by_tokens) gate[j] = of(b.gate, b.ld_gate);
      }
    }
  };
  auto fetch_late = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8, left = b.cols - c;
      if (a.ds) ds[j] = raw8_upto(static_cast<const T*>(a.ds) + row * a.ldds + c, left);
      if (by_tokens)
        gate[j] = raw8_upto(static_cast<const T*>(b.gate) + row * b.ld_gate + c, left);
    }
  };
  fetch(begin);
  for (int64_t row = begin; row < end; ++row) {
    const int odd = (row - begin) & 1;  // the sums alternate between two places
    float g[NV][8], hat[NV][8], z[NV][8], k[NV][8], both[2];
    const float d = rstd, pd = post_rstd;
    if constexpr (!HOLD) {
      parameter(b.weight, 0.0f, w);
      fetch_late(row);
    }
    both[0] = both[1] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t left = b.cols - (j * THREADS + threadIdx.x) * 8;
      unpack8<T>(dy[j], g[j]);
      unpack8<T>(s[j], hat[j]);
      unpack8<T>(h[j], z[j]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        hat[j][e] = (hat[j][e] - mean) * d;
        if (post) z[j][e] = (z[j][e] - post_mean) * pd;
        if (left < 8 && e >= left) hat[j][e] = z[j][e] = 0.0f;
      }
      add(0, j, g[j], hat[j]);
      if (HOLD || sums_of & 2) add(1, j, g[j], nullptr);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[j][e] *= w[j][e];
        both[0] += g[j][e];
        both[1] = __builtin_fmaf(g[j][e], hat[j][e], both[1]);
      }
    }
    // ds and the gate go on to the whole gradient, and the next row comes
    float more[NV][8];
    auto go_on = [&] {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        unpack8<T>(ds[j], more[j]);
        if (by_tokens) {
          unpack8<T>(gate[j], k[j]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) k[j][e] = gv[j][e];
        }
      }
    };
    if constexpr (HOLD) go_on();
    if (row + 1 < end) fetch(row + 1);
    if (a.dy) sums_group<kWaves, 2>(both, sums[0][odd]);
    if constexpr (!HOLD) {
      parameter(columns, 1.0f, gv);
      go_on();
      parameter(b.post_weight, 1.0f, pw);
      parameter(b.post_bias, 0.0f, pb);
    }
    const float along = b.rms || !a.dy ? 0.0f : both[0] * scale;
    const float across = a.dy ? both[1] * scale : 0.0f;
    both[0] = both[1] = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8, left = b.cols - c;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float v = more[j][e];
        if (a.dy) v += d * (g[j][e] - along - hat[j][e] * across);
        if (left < 8 && e >= left) v = 0.0f;
        g[j][e] = v;
        f[e] = post ? __builtin_fmaf(z[j][e], pw[j][e], pb[j][e]) : z[j][e];
        f[e] *= v;
        k[j][e] *= v;  // the gradient of N_post(h)
      }
      if (HOLD || sums_of & 4) add(2, j, k[j], z[j]);
      if (HOLD || sums_of & 8) add(3, j, k[j], nullptr);
      if (HOLD || sums_of & 16) add(4, j, f, nullptr);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        if (post) {
          k[j][e] *= pw[j][e];
          both[0] += k[j][e];
          both[1] = __builtin_fmaf(k[j][e], z[j][e], both[1]);
        }
        g[j][e] *= b.scale;
      }
      if (left > 0) {
        if (a.dx) store8_upto(static_cast<T*>(a.dx) + row * a.lddx + c, left, g[j]);
        if (a.dgate) store8_upto(static_cast<T*>(a.dgate) + row * a.lddgate + c, left, f);
      }
    }
    if (!a.dh) continue;
    if (post) sums_group<kWaves, 2>(both, sums[1][odd]);
    const float x = b.rms ? 0.0f : both[0] * scale, y = both[1] * scale;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8, left = b.cols - c;
      if (post) {
#pragma unroll
        for (int e = 0; e < 8; ++e) k[j][e] = pd * (k[j][e] - x - z[j][e] * y);
      }
      if (left > 0) store8_upto(static_cast<T*>(a.dh) + row * a.lddh + c, left, k[j]);
    }
  }
  int rank = 0;
  const int asked = __builtin_popcount(sums_of);
#pragma unroll
  for (int q = 0; q < kSums; ++q) {
    if (!(sums_of >> q & 1)) continue;
    float* out = partial + (static_cast<int64_t>(chunk) * asked + rank++) * b.cols;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int64_t c = (j * THREADS + threadIdx.x) * 8;
      if (c >= b.cols) continue;
      if (q < kHeld) {
        store8_upto(out + c, b.cols - c, total[q < kHeld ? q : 0][j]);
      } else {
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = totals[q - kHeld][j][e / 4][threadIdx.x][e % 4];
        store8_upto(out + c, b.cols - c, v);
      }
    }
  }
}

template <typename T>
__global__ __launch_bounds__(64) void k_residual_dw_long(ResidualNormBackward a, Chunks chunks,
                                                         const float2* means, int sums_of,
                                                         float* partial) {
  const int chunk = blockIdx.y, worker = worker_of(chunks, chunk);
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
  int rank = 0;
  const int asked = __builtin_popcount(sums_of);
#pragma unroll
  for (int q = 0; q < kSums; ++q)
    if (sums_of >> q & 1)
      store8_upto(partial + (static_cast<int64_t>(chunk) * asked + rank++) * a.b.cols + c,
                  a.b.cols - c, sum[q]);
}

// The chunks of a worker added in one order: 64 columns of one of the sums at a time for
// worker blockIdx.y, every fourth chunk to a wave.
__global__ __launch_bounds__(kBlock) void k_residual_sums(const float* __restrict__ partial,
                                                          int64_t cols, Chunks chunks, int sums_of,
                                                          garfield_residual_gradients to) {
  __shared__ float sums[4][64];
  const int asked = __builtin_popcount(sums_of);
  const int lane = threadIdx.x % 64, part = threadIdx.x / 64, worker = blockIdx.y;
  const int64_t groups = (cols + 63) / 64;
  for (int64_t i = blockIdx.x; i < groups * asked; i += gridDim.x) {
    const int rank = static_cast<int>(i / groups);
    const int64_t c = i % groups * 64 + lane;
    float sum = 0.0f;
    if (c < cols) {
#pragma unroll 8
      for (int k = chunks.chunk0[worker] + part; k < chunks.chunk0[worker + 1]; k += 4)
        sum += partial[(static_cast<int64_t>(k) * asked + rank) * cols + c];
    }
    sums[part][lane] = sum;
    __syncthreads();
    if (part == 0 && c < cols) {
      sum = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
      int q = 0;
      for (int left = rank; left >= 0; ++q) left -= sums_of >> q & 1;
      float* const outs[kSums] = {to.weight, to.bias, to.post_weight, to.post_bias, to.gate};
      const int64_t lds[kSums] = {to.ld_weight, to.ld_bias, to.ld_post_weight, to.ld_post_bias,
                                  to.ld_gate};
#pragma unroll
      for (int k = 0; k < kSums; ++k)
        if (k == q - 1) outs[k][worker * lds[k] + c] = sum;
    }
    __syncthreads();  // the sums' places are free
  }
}

int sums_asked(const garfield_residual_gradients& to) {
  return (to.weight ? 1 : 0) | (to.bias ? 2 : 0) | (to.post_weight ? 4 : 0) |
         (to.post_bias ? 8 : 0) | (to.gate ? 16 : 0);
}

constexpr int64_t kBackwardMaxCols = 8192;

template <typename T, int THREADS, int NV, bool HOLD = true>
void launch_backward(const ResidualNormBackward& a, const Chunks& c, float* partial, hipStream_t s) {
  launch("residual_backward", k_residual_backward<T, THREADS, NV, HOLD>, dim3(c.chunk0[c.n]),
         dim3(THREADS), 0, s, a, c, sums_asked(a.to), partial);
}

template <typename T>
void choose_backward(const ResidualNormBackward& a, const Chunks& c, void* workspace, hipStream_t s) {
  float2* means = static_cast<float2*>(workspace);
  const int64_t cols = a.b.cols;
  float* partial = reinterpret_cast<float*>(cols > kBackwardMaxCols ? means + a.b.rows : means);
  const int sums = sums_asked(a.to);
  if (a.b.rows > 0) {
    if (cols > kBackwardMaxCols) {
      launch("residual_dx_long", k_residual_dx_long<T>, dim3(static_cast<uint32_t>(a.b.rows)),
             dim3(kLong), 0, s, a, means);
      if (sums)
        launch("residual_dw_long", k_residual_dw_long<T>,
               dim3(static_cast<uint32_t>((cols + 511) / 512), c.chunk0[c.n]), dim3(64), 0, s, a, c,
               means, sums, partial);
    } else if (cols > 4096) {
      launch_backward<T, 512, 2, false>(a, c, partial, s);
    } else if (cols > 2048) {
      launch_backward<T, 512, 1>(a, c, partial, s);
    } else if (cols > 1024) {
      launch_backward<T, 256, 1>(a, c, partial, s);
    } else if (cols > 512) {
      launch_backward<T, 128, 1>(a, c, partial, s);
    } else {
      launch_backward<T, 64, 1>(a, c, partial, s);
    }
  }
  if (sums) {
    // a workgroup for 64 columns, up to 2^17 of them a worker: a launch has fewer than 2^32 threads
    const int64_t groups = (cols + 63) / 64 * __builtin_popcount(sums), most = int64_t{1} << 17;
    launch("residual_sums", k_residual_sums,
           dim3(static_cast<uint32_t>(groups < most ? groups : most), c.n), dim3(kBlock), 0, s,
           partial, cols, c, sums, a.to);
  }
}

template <typename T, int WAVES, int NV, int R>
void launch_forward(const ResidualNorm& a, hipStream_t s) {
  constexpr int kRows = WAVES > 4 ? R : 4 / WAVES * R;
  launch("residual_norm", k_residual_norm<T, WAVES, NV, R>,
         dim3(static_cast<uint32_t>((a.b.rows + kRows - 1) / kRows)),
         dim3(64 * (WAVES > 4 ? WAVES : 4)), 0, s, a);
}

// Two rows of more than 1024 columns at a time, or four narrow ones, where there are many: in
// bf16 131072 x 256 90 us, one at a time 110, 65536 x 768 94 and 121. A row of 4097 to 6144 columns
// has twelve waves (8192 x 5120 in fp32 144 us, in four with four vectors a lane 223).
template <typename T>
void choose_forward(const ResidualNorm& a, hipStream_t s) {
  const bool many = a.b.rows >= 8 * device_cus();
  const int64_t cols = a.b.cols;
  if (cols > 16384)
    launch("residual_norm_long", k_residual_norm_long<T>, dim3(static_cast<uint32_t>(a.b.rows)),
           dim3(kLong), 0, s, a);
  else if (cols > 8192) launch_forward<T, 16, 2, 1>(a, s);
  else if (cols > 6144) launch_forward<T, 8, 2, 1>(a, s);
  else if (cols > 4096) launch_forward<T, 12, 1, 1>(a, s);
  else if (many && cols > 2048) launch_forward<T, 4, 2, 2>(a, s);
  else if (many && cols > 1024) launch_forward<T, 4, 1, 2>(a, s);
  else if (cols > 2048) launch_forward<T, 4, 2, 1>(a, s);
  else if (cols > 1024) launch_forward<T, 4, 1, 1>(a, s);
  else if (many && cols > 512) launch_forward<T, 1, 2, 2>(a, s);
  else if (many) launch_forward<T, 1, 1, 4>(a, s);
  else if (cols > 512) launch_forward<T, 1, 2, 1>(a, s);
  else launch_forward<T, 1, 1, 1>(a, s);
}

}  // namespace

hipError_t enqueue_residual_norm(const ResidualNorm& a, hipStream_t s) {
  if (a.b.type == GARFIELD_F32) choose_forward<float>(a, s);
  else if (a.b.type == GARFIELD_BF16) choose_forward<__bf16>(a, s);
  else choose_forward<_Float16>(a, s);
  return hipGetLastError();
}

// Chunks of equal length, as many as the workgroups that the card holds at once and no more.
Chunks residual_norm_backward_chunks(const garfield_residual_block& b, int n,
                                     const int64_t* counts) {
  const int per_cu = b.cols > 2048 ? 1 : b.cols > 1024 ? 2 : b.cols > 512 ? 4 : 8;
  const int64_t want = static_cast<int64_t>(device_cus()) * per_cu;
  int64_t per = (b.rows + want - 1) / want;
  per = per < 2 ? 2 : per;
  Chunks c = make_chunks(n, counts, per);
  while (c.chunk0[n] > want && per < b.rows) {
    per += (per + 31) / 32;
    c = make_chunks(n, counts, per);
  }
  return c;
}

size_t residual_norm_backward_bytes(const garfield_residual_block& b, const Chunks& c) {
  const size_t means = b.cols > kBackwardMaxCols ? b.rows * sizeof(float2) : 0;
  return means + static_cast<size_t>(c.chunk0[c.n]) * kSums * b.cols * sizeof(float);
}

hipError_t enqueue_residual_norm_backward(const ResidualNormBackward& a, const Chunks& c,
                                          void* workspace, hipStream_t s) {
  if (a.b.type == GARFIELD_F32) choose_backward<float>(a, c, workspace, s);
  else if (a.b.type == GARFIELD_BF16) choose_backward<__bf16>(a, c, workspace, s);
  else choose_backward<_Float16>(a, c, workspace, s);
  return hipGetLastError();
}

}  // namespace garfield
