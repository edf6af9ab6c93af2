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

__device__ __forceinline__ float activate(int activation, float p) {
  switch (activation) {
    case GARFIELD_RELU: return p < 0.0f ? 0.0f : p;  // NaN stays
    case GARFIELD_GELU: return p * normal_below(p);
    case GARFIELD_GELU_TANH: return p * logistic(tanh_argument(p));
    case GARFIELD_SILU: return p * logistic(p);
    default: return p;
  }
}

__device__ __forceinline__ float slope(int activation, float p) {
  switch (activation) {
    case GARFIELD_RELU: return p > 0.0f ? 1.0f : 0.0f;
    case GARFIELD_GELU:
      return __builtin_fmaf(p * 0.39894228040143268f, expf(-0.5f * p * p), normal_below(p));
    case GARFIELD_GELU_TANH: {
      const float u = tanh_argument(p), q = logistic(u), rest = q * logistic(-u);
      const float du = kTanhScale * __builtin_fmaf(3.0f * kTanhCube * p, p, 1.0f);
      return rest == 0.0f ? q : __builtin_fmaf(p * rest, du, q);  // du may be infinite
    }
    case GARFIELD_SILU: {
      const float q = logistic(p);
      return q * __builtin_fmaf(p, logistic(-p), 1.0f);
    }
    default: return 1.0f;
  }
}

}  // namespace garfield
