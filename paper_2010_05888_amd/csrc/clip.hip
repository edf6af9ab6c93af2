// Each worker's gradient norm over many tensors, and its gradient clipped to a largest norm.
//
// Squares of fp32 values are exact in fp64 and cannot overflow there; their sums are added in
// one order: thread by thread, wave by wave, chunk by chunk.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

constexpr int64_t kChunk = 16384;  // values of a worker's tensor that a workgroup takes
constexpr int kTable = 64;         // tensors of a launch

// A launch's tensors, in its arguments. Workgroup g is of tensor i, first[i] <= g < first[i + 1].
struct Tensors {
  int count;
  uint32_t first[kTable + 1];
  garfield_gradient t[kTable];
  int64_t at[kTable];     // of the tensor in a worker's row of out
  int64_t chunk[kTable];  // its first chunk of a worker's
};

struct Part {
  int tensor, worker;
  int64_t chunk;  // of the tensor's row
};
__device__ __forceinline__ Part part_of(const Tensors& all, uint32_t g, uint32_t n) {
  int lo = 0, hi = all.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (all.first[mid] <= g) lo = mid;
    else hi = mid;
  }
  const uint32_t at = g - all.first[lo], rows = (all.first[lo + 1] - all.first[lo]) / n;
  return {lo, static_cast<int>(at / rows), static_cast<int64_t>(at % rows)};
}

__device__ __forceinline__ void load_any(const void* p, int type, int64_t i, int64_t left, float* v) {
  if (type == GARFIELD_F32) load8_upto(static_cast<const float*>(p) + i, left, v);
  else if (type == GARFIELD_BF16) load8_upto(static_cast<const __bf16*>(p) + i, left, v);
  else load8_upto(static_cast<const _Float16*>(p) + i, left, v);
}

__device__ __forceinline__ void store_any(void* p, int type, int64_t i, int64_t left, const float* v) {
  if (type == GARFIELD_F32) store8_upto(static_cast<float*>(p) + i, left, v);
  else if (type == GARFIELD_BF16) store8_upto(static_cast<__bf16*>(p) + i, left, v);
  else store8_upto(static_cast<_Float16*>(p) + i, left, v);
}

__device__ __forceinline__ double sum_block(double v) {
  __shared__ double at[kBlock / 64];
  v = sum_wave(v);
  if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
  __syncthreads();
  v = 0.0;
  for (int w = 0; w < kBlock / 64; ++w) v += at[w];
  return v;
}

// partial[worker][chunk], `chunks` of them a worker.
__global__ __launch_bounds__(kBlock) void k_squares(Tensors all, int n, int64_t chunks,
                                                    double* __restrict__ partial) {
  const Part p = part_of(all, blockIdx.x, n);
  const garfield_gradient t = all.t[p.tensor];
  const int64_t i0 = p.chunk * kChunk, end = i0 + kChunk < t.length ? i0 + kChunk : t.length;
  double sum = 0.0;
  for (int64_t i = i0 + threadIdx.x * 8; i < end; i += kBlock * 8) {
    float v[8];
    load_any(t.values, t.type, p.worker * t.ld + i, t.length - i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = __builtin_fma(static_cast<double>(v[e]), static_cast<double>(v[e]), sum);
  }
  sum = sum_block(sum);
  if (threadIdx.x == 0) partial[p.worker * chunks + all.chunk[p.tensor] + p.chunk] = sum;
}

__global__ __launch_bounds__(kBlock) void k_norms(const double* __restrict__ partial,
                                                  int64_t chunks, float max_norm,
                                                  float* __restrict__ norms,
                                                  float* __restrict__ factors) {
  double sum = 0.0;
  for (int64_t c = threadIdx.x; c < chunks; c += kBlock) sum += partial[blockIdx.x * chunks + c];
  const double norm = __builtin_sqrt(sum_block(sum)), most = max_norm;
  if (threadIdx.x == 0) {
    norms[blockIdx.x] = static_cast<float>(norm);
    factors[blockIdx.x] = norm <= most ? 1.0f : static_cast<float>(most / norm);  // NaN stays
  }
}

__global__ __launch_bounds__(kBlock) void k_scale(Tensors all, int n,
                                                  const float* __restrict__ factors,
                                                  float* __restrict__ out, int64_t ld_out) {
  const Part p = part_of(all, blockIdx.x, n);
  const garfield_gradient t = all.t[p.tensor];
  const float factor = factors[p.worker];
  if (!out && factor == 1.0f) return;
  const int64_t i0 = p.chunk * kChunk, end = i0 + kChunk < t.length ? i0 + kChunk : t.length;
  for (int64_t i = i0 + threadIdx.x * 8; i < end; i += kBlock * 8) {
    float v[8];
    load_any(t.values, t.type, p.worker * t.ld + i, t.length - i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= factor;
    if (out) store8_upto(out + p.worker * ld_out + all.at[p.tensor] + i, t.length - i, v);
    else store_any(t.values, t.type, p.worker * t.ld + i, t.length - i, v);
  }
}

int64_t chunks_of(const garfield_gradient& t) { return (t.length + kChunk - 1) / kChunk; }

// f(tensors, workgroups) for every launch that has work: as many tensors as its arguments hold,
// and no more workgroups than a launch has.
template <class F>
void for_each_launch(const garfield_gradient* tensors, int count, int n, F&& f) {
  constexpr int64_t kMost = 0xffffffff / kBlock;
  Tensors all = {};
  int64_t at = 0, chunk = 0, groups = 0;
  for (int i = 0; i < count; ++i) {
    const int64_t chunks = chunks_of(tensors[i]);
    if (chunks == 0) continue;
    // a tensor of more chunks than a launch takes is cut (its rows are cut alike)
    for (int64_t c = 0; c < chunks;) {
      if (all.count == kTable || groups + n > kMost) {
        f(all, groups);
        all.count = 0;
        groups = 0;
      }
      const int64_t room = (kMost - groups) / n;
      const int64_t some = chunks - c < room ? chunks - c : room;
      garfield_gradient t = tensors[i];
      const int64_t skipped = c * kChunk;
      t.values = static_cast<char*>(t.values) + skipped * (t.type == GARFIELD_F32 ? 4 : 2);
      t.length = c + some == chunks ? t.length - skipped : some * kChunk;
      all.t[all.count] = t;
      all.at[all.count] = at + skipped;
      all.chunk[all.count] = chunk + c;
      all.first[all.count] = static_cast<uint32_t>(groups);
      groups += some * n;
      all.first[++all.count] = static_cast<uint32_t>(groups);
      c += some;
    }
    at += tensors[i].length;
    chunk += chunks;
  }
  if (all.count > 0) f(all, groups);
}

}  // namespace

size_t clip_bytes(const garfield_gradient* tensors, int count, int n) {
  int64_t chunks = 0;
  for (int i = 0; i < count; ++i) chunks += chunks_of(tensors[i]);
  return static_cast<size_t>(n) * (chunks * sizeof(double) + sizeof(float));
}

hipError_t enqueue_clip(const garfield_gradient* tensors, int count, int n, float max_norm,
                        float* norms, float* out, int64_t ld_out, void* workspace, hipStream_t s) {
  int64_t chunks = 0;
  for (int i = 0; i < count; ++i) chunks += chunks_of(tensors[i]);
  double* partial = static_cast<double*>(workspace);
  float* factors = reinterpret_cast<float*>(partial + n * chunks);
  for_each_launch(tensors, count, n, [&](const Tensors& all, int64_t groups) {
    launch("squares", k_squares, dim3(static_cast<uint32_t>(groups)), dim3(kBlock), 0, s, all, n,
           chunks, partial);
  });
  launch("norms", k_norms, dim3(n), dim3(kBlock), 0, s, partial, chunks, max_norm, norms, factors);
  if (max_norm == max_norm)
    for_each_launch(tensors, count, n, [&](const Tensors& all, int64_t groups) {
      launch("scale", k_scale, dim3(static_cast<uint32_t>(groups)), dim3(kBlock), 0, s, all, n,
             factors, out, ld_out);
    });
  return hipGetLastError();
}

}  // namespace garfield
