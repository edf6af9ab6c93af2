// A linear layer's activations and their slopes, in fp32.
//
// Each is written so that no difference of nearly equal values loses its digits: gelu's
// Phi(p) = erfc(-p / sqrt(2)) / 2 also where it is small, and the others by the logistic
// function, q(u) = 1 / (1 + exp(-u)): silu is p q(p), and (1 + tanh(v)) / 2 = q(2 v).
#pragma once

#include <hip/hip_runtime.h>

#include "garfield_worker.h"

namespace garfield {

__device__ __forceinline__ float logistic(float u) { return 1.0f / (1.0f + expf(-u)); }

// 2 sqrt(2 / pi) (p + 0.044715 p^3) and its slope.
constexpr float kTanhScale = 1.5957691216057308f, kTanhCube = 0.044715f;
__device__ __forceinline__ float tanh_argument(float p) {
  return kTanhScale * p * __builtin_fmaf(kTanhCube * p, p, 1.0f);
}

__device__ __forceinline__ float normal_below(float p) {
  return 0.5f * erfcf(-0.70710678118654752f * p);
}

// N values at a time, for one decision.
template <int N>
__device__ __forceinline__ void activate(int activation, float* v) {
  switch (activation) {
    case GARFIELD_RELU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = v[e] < 0.0f ? 0.0f : v[e];  // NaN stays
      break;
    case GARFIELD_GELU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= normal_below(v[e]);
      break;
    case GARFIELD_GELU_TANH:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= logistic(tanh_argument(v[e]));
      break;
    case GARFIELD_SILU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= logistic(v[e]);
      break;
    default: break;
  }
}

__device__ __forceinline__ float gelu_slope(float p) {
  return __builtin_fmaf(p * 0.39894228040143268f, expf(-0.5f * p * p), normal_below(p));
}

__device__ __forceinline__ float gelu_tanh_slope(float p) {
  const float u = tanh_argument(p), q = logistic(u), rest = q * logistic(-u);
  const float du = kTanhScale * __builtin_fmaf(3.0f * kTanhCube * p, p, 1.0f);
  return rest == 0.0f ? q : __builtin_fmaf(p * rest, du, q);  // du may be infinite
}

// v times the slopes at p.
template <int N>
__device__ __forceinline__ void times_slope(int activation, const float* p, float* v) {
  switch (activation) {
    case GARFIELD_RELU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= p[e] > 0.0f ? 1.0f : 0.0f;
      break;
    case GARFIELD_GELU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= gelu_slope(p[e]);
      break;
    case GARFIELD_GELU_TANH:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= gelu_tanh_slope(p[e]);
      break;
    case GARFIELD_SILU:
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float q = logistic(p[e]);
        v[e] *= q * __builtin_fmaf(p[e], logistic(-p[e]), 1.0f);
      }
      break;
    default: break;
  }
}

}  // namespace garfield
