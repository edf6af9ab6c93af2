// A linear layer's activations and their slopes, in fp32.
//
// Each is p q(u), with the logistic function q(u) = 1 / (1 + exp(-u)) and u odd in p: silu has
// u = p, gelu's approximation by tanh u = 2 sqrt(2 / pi) (p + 0.044715 p^3), for (1 + tanh(v)) / 2
// = q(2 v), and gelu itself u = log(Phi(p) / Phi(-p)), which is p times a polynomial in p^2 to
// what fp32 shows. One exponential and one reciprocal, each off by a unit or so in the last
// place, make p q(u) right to 3 u (1 + |p|), u = 2^-24, and gelu's small values at p < 0 to 2^-13
// of themselves down to p = -6, where they are 6e-9; q below 2^-126 is 0. A product's epilogue has
// no time to spare: with 134 million outputs gelu by erfc took 91 us more than this does.
#pragma once

#include <hip/hip_runtime.h>

#include "garfield_worker.h"

namespace garfield {

constexpr float kLog2e = 1.4426950408889634f;

// exp(-u), and q(u), of u * log2(e).
__device__ __forceinline__ float exp_minus(float u) { return __builtin_amdgcn_exp2f(-u); }
__device__ __forceinline__ float logistic(float e) { return __builtin_amdgcn_rcpf(1.0f + e); }

// log2(e) log(Phi(p) / Phi(-p)): p times a polynomial in p^2 up to 36 of least largest error,
// weighted for p Phi(p) (the polynomial's value at 36 beyond: q is 1e-9 there).
__device__ __forceinline__ float normal_argument(float p) {
  const float s = __builtin_fminf(p * p, 36.0f);
  float v = 1.1242183399484684e-12f;
  v = __builtin_fmaf(v, s, -1.918764452879529e-10f);
  v = __builtin_fmaf(v, s, 1.3896963579895782e-08f);
  v = __builtin_fmaf(v, s, -5.547715886677906e-07f);
  v = __builtin_fmaf(v, s, 1.3082096302241553e-05f);
  v = __builtin_fmaf(v, s, -0.00016725389286875725f);
  v = __builtin_fmaf(v, s, -7.726704643573612e-05f);
  v = __builtin_fmaf(v, s, 0.10482028126716614f);
  v = __builtin_fmaf(v, s, 2.302212953567505f);
  return p * v;
}

// The same for gelu's approximation by tanh.
constexpr float kTanhScale = kLog2e * 1.5957691216057308f, kTanhCube = 0.044715f;
__device__ __forceinline__ float tanh_argument(float p) {
  return p * __builtin_fmaf(p * p, kTanhScale * kTanhCube, kTanhScale);
}

__device__ __forceinline__ float clamped(float p, float to) {
  return p != p ? p : __builtin_amdgcn_fmed3f(p, -to, to);  // NaN stays
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
      for (int e = 0; e < N; ++e) v[e] *= logistic(exp_minus(normal_argument(v[e])));
      break;
    case GARFIELD_GELU_TANH:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= logistic(exp_minus(tanh_argument(v[e])));
      break;
    case GARFIELD_SILU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] *= logistic(exp_minus(kLog2e * v[e]));
      break;
    default: break;
  }
}

// (p q(u))' = q + p u' q (1 - q), 1 - q = e q. p is kept where e and p u' are finite; beyond
// that the slopes are 0 and 1. gelu's p, of which only an infinite one must not meet the density's
// 0, is kept to 1e18, far beyond where the density is 0; the density's factor (2 pi)^(-1/2) is in
// its exponent, which makes up for that instruction.
__device__ __forceinline__ float gelu_slope(float p) {
  const float density =
      __builtin_amdgcn_exp2f(__builtin_fmaf(p * p, -0.5f * kLog2e, -1.3257480647361592f));
  return __builtin_fmaf(__builtin_amdgcn_fmed3f(p, -1e18f, 1e18f), density,
                        logistic(exp_minus(normal_argument(p))));
}

__device__ __forceinline__ float gelu_tanh_slope(float p) {
  p = clamped(p, 10.0f);
  const float e = exp_minus(tanh_argument(p)), q = logistic(e);
  const float du = __builtin_fmaf(p * p, 3.0f * 1.5957691216057308f * kTanhCube, 1.5957691216057308f);
  return __builtin_fmaf(p * du, e * q * q, q);
}

__device__ __forceinline__ float silu_slope(float p) {
  p = clamped(p, 80.0f);
  const float e = exp_minus(kLog2e * p), q = logistic(e);
  return __builtin_fmaf(p, e * q * q, q);
}

// v times the slopes at p; relu's is 0 or 1, and chosen: where it is 0 nothing of v gets on, not an
// infinity either.
template <int N>
__device__ __forceinline__ void times_slope(int activation, const float* p, float* v) {
  switch (activation) {
    case GARFIELD_RELU:
#pragma unroll
      for (int e = 0; e < N; ++e) v[e] = p[e] > 0.0f ? v[e] : 0.0f;
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
      for (int e = 0; e < N; ++e) v[e] *= silu_slope(p[e]);
      break;
    default: break;
  }
}

}  // namespace garfield
