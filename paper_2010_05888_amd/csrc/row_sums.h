// What the norms of rows share: sums over a workgroup, the exact mean's lanes, weights, and a
// row's 8-bit blocks.
#pragma once

#include "block8.h"
#include "worker.h"

namespace garfield {

// Sum over the workgroup of `waves` waves; the same value in every thread.
// `at` holds one value a wave and is free again after the next barrier.
template <int WAVES, typename F>
__device__ __forceinline__ F sum_group(F v, F* at) {
  v = sum_wave(v);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) v += at[w];
  }
  return v;
}

// The same of R values, with one barrier for all. `at` holds R values a wave.
template <int WAVES, int R, typename F>
__device__ __forceinline__ void sums_group(F* v, F (*at)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = sum_wave(v[r]);
  if constexpr (WAVES > 1) {
    if (threadIdx.x % 64 == 0) {
#pragma unroll
      for (int r = 0; r < R; ++r) at[threadIdx.x / 64][r] = v[r];
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      v[r] = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) v[r] += at[w][r];
    }
  }
}

// What a lane adds up for the mean: the differences to its own first value, which are exact
// or nearly so where a row lies far from 0, and that value as often in fp64. An error of
// the mean is one of every value of the row: with plain fp32 sums a row of equal values
// -9999.9 had results up to 0.3 instead of 0. (8192 x 2048 in bf16 with y8 takes 18.2 us so and
// 17.7 with those, 65536 x 4096 197 and 196, 8192 x 16384 137 and 132.) The first value is
// taken as 0 if it is not finite, or so large that a difference could be infinite.
__device__ __forceinline__ float first_value(float v) {
  return __builtin_fabsf(v) < 0x1p102f ? v : 0.0f;
}
__device__ __forceinline__ double lane_total(float first, int count, float differences) {
  return __builtin_fma(static_cast<double>(first), static_cast<double>(count),
                       static_cast<double>(differences));
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
  const int s = block_shift(max16(largest<8>(v)));
  const int64_t blocks = (out.cols + kBlock8 - 1) / kBlock8;
  const int64_t b = c / kBlock8;
  if (b < blocks)
    *reinterpret_cast<u2*>(out.values + row * out.ld_values + c) = encode8(v, s);
  if (c % kBlock8 == 0 && b < (blocks + 3) / 4 * 4)
    out.exponents[row * out.ld_exponents + b] = static_cast<uint8_t>(b < blocks ? s + 127 : 127);
}

// The worker whose chunk it is: as many workers end at or before it.
__device__ __forceinline__ int worker_of(const Chunks& c, int chunk) {
  const int lane = threadIdx.x % 64;
  static_assert(kWorkersMax == 64, "a lane looks at one worker");
  return __builtin_popcountll(__ballot(lane < c.n && c.chunk0[lane + 1] <= chunk));
}

}  // namespace garfield
