// Each worker's gradient norm over many tensors, and its gradient clipped to a largest norm.
//
// Squares of fp32 values are exact in fp64 and cannot overflow there; their sums are added in
// one order: lane by lane, wave by wave, chunk by chunk.
//
// Bound by memory: a value is read for the norm, and read and written for its clipped one. 19
// workers' 25,557,032 values in 161 tensors take 350 us for the norms (5.5 TB/s) and 777 for the
// rest (5.0, as a copy). 11 workers' 100,000 values take 3.8 + 5.6 us, latency. The norm comes
// first, and a worker's row is behind the caches when it is known: taking the workers one after the
// other, 102 MB each, was no faster (1339 against 1115 us).

#include <algorithm>

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

constexpr int kTable = 64;  // tensors in a launch's arguments

// A tensor, where it goes in a worker's row of the result, and the chunks before it.
struct Entry {
  garfield_gradient t;
  int64_t at, chunk;
};
struct Table {
  int count;
  Entry e[kTable];
};

// Tables of more tensors than that are put together in the workspace.
__global__ __launch_bounds__(kTable) void k_table(Table part, Entry* __restrict__ to) {
  if (static_cast<int>(threadIdx.x) < part.count) to[threadIdx.x] = part.e[threadIdx.x];
}

// The tensor whose chunk it is; `e` in memory or in the arguments. Up to 256 are looked at at
// once, more one after the other.
template <typename Entries>
__device__ __forceinline__ int tensor_of(const Entries& e, int count, int64_t chunk) {
  if (count <= 256) {
    int at_or_before = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = k * 64 + threadIdx.x % 64;
      if (k * 64 < count)
        at_or_before += __builtin_popcountll(__ballot(i < count && e[i < count ? i : 0].chunk <= chunk));
    }
    return __builtin_amdgcn_readfirstlane(at_or_before) - 1;
  }
  int lo = 0, hi = count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (e[mid].chunk <= chunk) lo = mid;
    else hi = mid;
  }
  return lo;
}

// v's eight values squared and added.
template <typename T>
__device__ __forceinline__ double add_squares(const typename Pack8<T>::type& v, double sum) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const double x = static_cast<double>(static_cast<float>(v[e]));
    sum = __builtin_fma(x, x, sum);
  }
  return sum;
}

// Values before the first address that is a multiple of 32 bytes, fewer than 16: a worker's row
// of a tensor starts anywhere.
template <typename T>
__device__ __forceinline__ int64_t before_line(const T* p, int64_t length) {
  const int64_t n = (32 - reinterpret_cast<uintptr_t>(p) % 32) % 32 / sizeof(T);
  return n < length ? n : length;
}

// A thread's part of a chunk: four vectors at a time on their way, at its end too (one by one
// there, the norms took 365 us).
template <typename T>
__device__ __forceinline__ double chunk_squares(const T* p, int64_t length) {
  constexpr int64_t kApart = kBlock * 8;
  double sum = 0.0;
  const int64_t head = before_line(p, length);
  if (threadIdx.x < head) {
    const double x = static_cast<double>(static_cast<float>(p[threadIdx.x]));
    sum = x * x;
  }
  p += head;
  length -= head;
  int64_t i = threadIdx.x * 8;
  for (; i - threadIdx.x * 8 + kApart < length; i += 4 * kApart) {
    typename Pack8<T>::type v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = raw8_upto(p + i + k * kApart, length - i - k * kApart);
#pragma unroll
    for (int k = 0; k < 4; ++k) sum = add_squares<T>(v[k], sum);
  }
  if (i < length) sum = add_squares<T>(raw8_upto(p + i, length - i), sum);
  return sum;
}

template <typename T, typename Out>
__device__ __forceinline__ void chunk_scale(const T* p, int64_t length, float factor, Out* out) {
  constexpr int64_t kApart = kBlock * 8;
  const int64_t head = before_line(out, length);  // whole lines are written
  if (threadIdx.x < head)
    out[threadIdx.x] = static_cast<Out>(static_cast<float>(p[threadIdx.x]) * factor);
  p += head;
  out += head;
  length -= head;
  int64_t i = threadIdx.x * 8;
  float t[8];
  for (; i - threadIdx.x * 8 + kApart < length; i += 4 * kApart) {
    typename Pack8<T>::type v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = raw8_upto(p + i + k * kApart, length - i - k * kApart);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      unpack8<T>(v[k], t);
#pragma unroll
      for (int e = 0; e < 8; ++e) t[e] *= factor;
      store8_upto(out + i + k * kApart, length - i - k * kApart, t);
    }
  }
  if (i < length) {
    load8_upto(p + i, length - i, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= factor;
    store8_upto(out + i, length - i, t);
  }
}

// f(values of the tensor's type)
template <typename F>
__device__ __forceinline__ void by_type(void* p, int type, F&& f) {
  if (type == GARFIELD_F32) f(static_cast<float*>(p));
  else if (type == GARFIELD_BF16) f(static_cast<__bf16*>(p));
  else f(static_cast<_Float16*>(p));
}

template <int WAVES>
__device__ __forceinline__ double sum_block(double v, double* at) {
  v = sum_wave(v);
  if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) v += at[w];
  __syncthreads();
  return v;
}

__device__ __forceinline__ float factor_of(double norm, float max_norm) {
  const double most = max_norm;
  return norm <= most ? 1.0f : static_cast<float>(most / norm);  // NaN stays
}

// partial[worker][chunk], `chunks` of them a worker.
template <bool MEMORY>
__global__ __launch_bounds__(kBlock) void k_squares(Table table, const Entry* __restrict__ more,
                                                    int count, int n, int64_t chunks,
                                                    int64_t length,
                                                    double* __restrict__ partial) {
  __shared__ double at[kBlock / 64];
  for (int64_t b = blockIdx.x; b < n * chunks; b += gridDim.x) {
    const int64_t worker = b / chunks, chunk = b % chunks;
    const Entry e = MEMORY ? more[tensor_of(more, count, chunk)]
                           : table.e[tensor_of(table.e, count, chunk)];
    const int64_t first = (chunk - e.chunk) * length, left = e.t.length - first;
    double sum = 0.0;
    by_type(e.t.values, e.t.type, [&](auto* p) {
      sum = chunk_squares(p + worker * e.t.ld + first, left < length ? left : length);
    });
    sum = sum_block<kBlock / 64>(sum, at);
    if (threadIdx.x == 0) partial[b] = sum;
  }
}

__global__ __launch_bounds__(kBlock) void k_norms(const double* __restrict__ partial,
                                                  int64_t chunks, float max_norm,
                                                  float* __restrict__ norms,
                                                  float* __restrict__ factors) {
  __shared__ double at[kBlock / 64];
  double sum = 0.0;
#pragma unroll 4
  for (int64_t c = threadIdx.x; c < chunks; c += kBlock) sum += partial[blockIdx.x * chunks + c];
  const double norm = __builtin_sqrt(sum_block<kBlock / 64>(sum, at));
  if (threadIdx.x == 0) {
    norms[blockIdx.x] = static_cast<float>(norm);
    factors[blockIdx.x] = factor_of(norm, max_norm);
  }
}

// A worker's norm from few chunks is added up by each of its workgroups, and no launch of its own.
constexpr int64_t kOwnSum = 4 * kBlock;

template <bool MEMORY>
__global__ __launch_bounds__(kBlock) void k_scale(Table table, const Entry* __restrict__ more,
                                                  int count, int n, int64_t chunks,
                                                  int64_t most,
                                                  const double* __restrict__ partial,
                                                  float max_norm, float* __restrict__ norms,
                                                  const float* __restrict__ factors,
                                                  float* __restrict__ out, int64_t ld_out) {
  __shared__ double at[kBlock / 64];
  for (int64_t b = blockIdx.x; b < n * chunks; b += gridDim.x) {
    const int64_t worker = b / chunks, chunk = b % chunks;
    float factor;
    if (chunks <= kOwnSum) {
      double sum = 0.0;
#pragma unroll
      for (int k = 0; k < kOwnSum / kBlock; ++k) {
        const int64_t c = k * kBlock + threadIdx.x;
        if (c < chunks) sum += partial[worker * chunks + c];
      }
      const double norm = __builtin_sqrt(sum_block<kBlock / 64>(sum, at));
      factor = factor_of(norm, max_norm);
      if (chunk == 0 && threadIdx.x == 0) norms[worker] = static_cast<float>(norm);
    } else {
      factor = factors[worker];
    }
    if (!out && factor == 1.0f) continue;
    const Entry e = MEMORY ? more[tensor_of(more, count, chunk)]
                           : table.e[tensor_of(table.e, count, chunk)];
    const int64_t first = (chunk - e.chunk) * most, left = e.t.length - first;
    const int64_t length = left < most ? left : most;
    by_type(e.t.values, e.t.type, [&](auto* p) {
      p += worker * e.t.ld + first;
      if (out) chunk_scale(p, length, factor, out + worker * ld_out + e.at + first);
      else chunk_scale(p, length, factor, p);
    });
  }
}

// All of it in one launch, a workgroup a worker, where a worker has few values of one type: its
// waves take chunks of 512 in turn, four at a time on their way, and read them again when the
// norm is known. (A CU has no more than some 60 GB/s so: 11 workers' 100,000 values take 20 us.)
constexpr int64_t kFew = 16384;
constexpr int kFewWaves = 16;
struct FewTable {
  int count;
  int first[kTable + 1];  // chunks of 512 before each tensor
  garfield_gradient t[kTable];
  int64_t at[kTable];
};
template <typename T>
__global__ __launch_bounds__(64 * kFewWaves) void k_clip_few(FewTable table, float max_norm,
                                                             float* __restrict__ norms,
                                                             float* out, int64_t ld_out,
                                                             bool norms_alone) {
  constexpr int kAtOnce = 4;
  __shared__ double at[kFewWaves];
  const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int64_t worker = blockIdx.x;
  const int chunks = table.first[table.count];
  // f(tensor, the lane's first value of a chunk, how many are there from it on, eight of them)
  auto each = [&](auto&& f) {
    int tensor = 0;
    for (int c0 = wave; c0 < chunks; c0 += kFewWaves * kAtOnce) {
      typename Pack8<T>::type v[kAtOnce];
      int of[kAtOnce], from[kAtOnce], left[kAtOnce];
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) {
        const int c = c0 + k * kFewWaves < chunks ? c0 + k * kFewWaves : chunks - 1;
        while (c >= table.first[tensor + 1]) ++tensor;
        const garfield_gradient& t = table.t[tensor];
        of[k] = tensor;
        from[k] = (c - table.first[tensor]) * 512 + lane * 8;
        left[k] = c == c0 + k * kFewWaves ? static_cast<int>(t.length) - from[k] : 0;
        v[k] = raw8_upto(static_cast<const T*>(t.values) + worker * t.ld + from[k], left[k]);
      }
#pragma unroll
      for (int k = 0; k < kAtOnce; ++k) f(of[k], from[k], left[k], v[k]);
    }
  };
  double sum = 0.0;
  each([&](int, int, int, const typename Pack8<T>::type& v) { sum = add_squares<T>(v, sum); });
  const double norm = __builtin_sqrt(sum_block<kFewWaves>(sum, at));
  if (threadIdx.x == 0) norms[worker] = static_cast<float>(norm);
  const float factor = factor_of(norm, max_norm);
  if (norms_alone || (!out && factor == 1.0f)) return;
  each([&](int tensor, int from, int left, const typename Pack8<T>::type& v) {
    float t[8];
    unpack8<T>(v, t);
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] *= factor;
    if (out)
      store8_upto(out + worker * ld_out + table.at[tensor] + from, left, t);
    else
      store8_upto(static_cast<T*>(table.t[tensor].values) + worker * table.t[tensor].ld + from, left,
                  t);
  });
}

int64_t chunks_of(const garfield_gradient& t, int64_t length) {
  return (t.length + length - 1) / length;
}

// Tensors that hold values, a worker's values, their type (-1: several), and the chunks.
struct Totals {
  int count, type;
  int64_t values, length, chunks;  // length: of a chunk
};
Totals totals(const garfield_gradient* tensors, int count, int n) {
  Totals all = {};
  for (int i = 0; i < count; ++i) {
    if (tensors[i].length == 0) continue;
    all.type = all.count == 0 || all.type == tensors[i].type ? tensors[i].type : -1;
    ++all.count;
    all.values += tensors[i].length;
  }
  // as long as there are four chunks for a CU, up to 16384 (chunks of 65536: 19 workers'
  // 25,557,032 values 45 us more)
  all.length = 16384;
  while (all.length > 2048 && n * all.values < all.length * 4 * device_cus()) all.length /= 2;
  for (int i = 0; i < count; ++i) all.chunks += chunks_of(tensors[i], all.length);
  return all;
}

bool is_few(const Totals& all) {
  return all.count <= kTable && all.values <= kFew && all.type >= 0;
}

}  // namespace

size_t clip_bytes(const garfield_gradient* tensors, int count, int n) {
  const Totals all = totals(tensors, count, n);
  if (is_few(all)) return 0;
  return static_cast<size_t>(n) * all.chunks * sizeof(double) +
         (all.count > kTable ? all.count * sizeof(Entry) : 0) + n * sizeof(float);
}

hipError_t enqueue_clip(const garfield_gradient* tensors, int count, int n, float max_norm,
                        float* norms, float* out, int64_t ld_out, void* workspace, hipStream_t s) {
  const Totals all = totals(tensors, count, n);
  const bool norms_alone = max_norm != max_norm;
  if (is_few(all)) {
    FewTable few = {};
    int64_t at = 0;
    for (int i = 0; i < count; ++i) {
      if (tensors[i].length == 0) continue;
      const int k = few.count++;
      few.t[k] = tensors[i];
      few.at[k] = at;
      few.first[k + 1] = few.first[k] + static_cast<int>((tensors[i].length + 511) / 512);
      at += tensors[i].length;
    }
    launch("clip_few",
           all.type == GARFIELD_F32    ? k_clip_few<float>
           : all.type == GARFIELD_BF16 ? k_clip_few<__bf16>
                                       : k_clip_few<_Float16>,
           dim3(n), dim3(64 * kFewWaves), 0, s, few, max_norm, norms, out, ld_out, norms_alone);
    return hipGetLastError();
  }
  double* partial = static_cast<double*>(workspace);
  Entry* more = reinterpret_cast<Entry*>(partial + n * all.chunks);
  float* factors = reinterpret_cast<float*>(all.count > kTable ? more + all.count : more);
  Table table = {};
  int written = 0;
  int64_t at = 0, chunk = 0;
  auto flush = [&] {
    launch("table", k_table, dim3(1), dim3(kTable), 0, s, table, more + written);
    written += table.count;
    table.count = 0;
  };
  for (int i = 0; i < count; ++i) {
    if (tensors[i].length == 0) continue;
    if (table.count == kTable) flush();
    table.e[table.count++] = {tensors[i], at, chunk};
    at += tensors[i].length;
    chunk += chunks_of(tensors[i], all.length);
  }
  const bool memory = all.count > kTable;
  if (memory && table.count > 0) flush();
  // a launch has fewer than 2^32 threads
  const int64_t groups = std::min(n * all.chunks, int64_t{1} << 23);
  const dim3 grid(static_cast<uint32_t>(groups));
  launch("squares", memory ? k_squares<true> : k_squares<false>, grid, dim3(kBlock), 0, s, table,
         static_cast<const Entry*>(more), all.count, n, all.chunks, all.length, partial);
  if (norms_alone || all.chunks > kOwnSum)
    launch("norms", k_norms, dim3(n), dim3(kBlock), 0, s, static_cast<const double*>(partial),
           all.chunks, max_norm, norms, factors);
  if (!norms_alone)
    launch("scale", memory ? k_scale<true> : k_scale<false>, grid, dim3(kBlock), 0, s, table,
           static_cast<const Entry*>(more), all.count, n, all.chunks, all.length,
           static_cast<const double*>(partial), max_norm, norms,
           static_cast<const float*>(factors), out, ld_out);
  return hipGetLastError();
}

}  // namespace garfield
