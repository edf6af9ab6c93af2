// Element types and 8-bit blocks on the device. A block is 128 values of a row:
// e4m3 codes and one exponent s, the smallest with max |v| <= 448 * 2^s (at
// least -117). 2^s is a power of two, so a code depends on its block's input
// bits alone and code * 2^s is exact in bf16 (4 significant bits, and no
// subnormal: the smallest is 2^-9 * 2^-117).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace garfield {

constexpr int kBlock8 = 128;
constexpr int kMinShift = -117;

typedef int i8v __attribute__((ext_vector_type(8)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

// Eight elements at the alignment of one: global memory serves 16-byte
// accesses at any address, so rows of any length and start are read with them.
template <typename T>
struct Pack8 {
  typedef T type __attribute__((ext_vector_type(8), aligned(sizeof(T))));
};

template <typename T>
__device__ __forceinline__ void unpack8(const typename Pack8<T>::type& t, float* v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(t[e]);
}

// The first `left` of eight elements as they are; the others 0.
template <typename T>
__device__ __forceinline__ typename Pack8<T>::type raw8_upto(const T* p, int64_t left) {
  if (left >= 8) return *reinterpret_cast<const typename Pack8<T>::type*>(p);
  typename Pack8<T>::type t;
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = static_cast<T>(0.0f);
  if (left > 0) {  // lanes past the row's end are many, and pass by
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) t[e] = p[e];
  }
  return t;
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* v) {
  const auto t = *reinterpret_cast<const typename Pack8<T>::type*>(p);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(t[e]);
}

// The first `left` of eight elements; the others read as 0.
template <typename T>
__device__ __forceinline__ void load8_tail(const T* p, int64_t left, float* v) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.0f;
  if (left > 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) v[e] = static_cast<float>(p[e]);
  }
}

template <typename T>
__device__ __forceinline__ void load8_upto(const T* p, int64_t left, float* v) {
  if (left >= 8) load8(p, v);
  else load8_tail(p, left, v);
}

template <typename T>
__device__ __forceinline__ void store8_upto(T* p, int64_t left, const float* v) {
  if (left >= 8) {
    typename Pack8<T>::type t;
#pragma unroll
    for (int e = 0; e < 8; ++e) t[e] = static_cast<T>(v[e]);
    *reinterpret_cast<typename Pack8<T>::type*>(p) = t;
  } else if (left > 0) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < left) p[e] = static_cast<T>(v[e]);
  }
}

// Rotate within the wave's rows of 16 lanes.
template <int BY>
__device__ __forceinline__ float row_ror(float v) {
  return __int_as_float(
      __builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x120 + BY, 0xf, 0xf, false));
}

// Over 16 lanes (a block's, eight values each); every lane gets the result.
__device__ __forceinline__ float max16(float v) {
  v = __builtin_fmaxf(v, row_ror<8>(v));
  v = __builtin_fmaxf(v, row_ror<4>(v));
  v = __builtin_fmaxf(v, row_ror<2>(v));
  return __builtin_fmaxf(v, row_ror<1>(v));
}

__device__ __forceinline__ float sum16(float v) {
  v += row_ror<8>(v);
  v += row_ror<4>(v);
  v += row_ror<2>(v);
  return v + row_ror<1>(v);
}

__device__ __forceinline__ float read_lane(float v, int lane) {
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// Over the wave, in one order for every lane.
__device__ __forceinline__ float sum_wave(float v) {
  v = sum16(v);
  return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}

// The same in 64 bits.
template <int BY>
__device__ __forceinline__ double row_ror(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(b), 0x120 + BY, 0xf, 0xf, false);
  const uint32_t hi =
      __builtin_amdgcn_update_dpp(0, static_cast<int>(b >> 32), 0x120 + BY, 0xf, 0xf, false);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}

__device__ __forceinline__ double read_lane(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}

__device__ __forceinline__ double sum_wave(double v) {
  v += row_ror<8>(v);
  v += row_ror<4>(v);
  v += row_ror<2>(v);
  v += row_ror<1>(v);
  return (read_lane(v, 0) + read_lane(v, 16)) + (read_lane(v, 32) + read_lane(v, 48));
}

__device__ __forceinline__ bool finite(float v) {
  return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
}

// The largest finite magnitude of N values. A maximum passes NaN over by itself, so
// only an infinite one is looked for again.
template <int N>
__device__ __forceinline__ float largest(const float* v) {
  float a = 0.0f;
#pragma unroll
  for (int e = 0; e < N; ++e) a = __builtin_fmaxf(a, __builtin_fabsf(v[e]));
  if (!finite(a)) {
    a = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) a = __builtin_fmaxf(a, finite(v[e]) ? __builtin_fabsf(v[e]) : 0.0f);
  }
  return a;
}

// s of a block whose largest finite magnitude is a. 448 = 1.75 * 2^8: with
// a = m * 2^k, s = k - 8 if m <= 1.75, else k - 7.
__device__ __forceinline__ int block_shift(float a) {
  const uint32_t b = __float_as_uint(a);
  const int s = static_cast<int>(b >> 23) - 127 - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return s > kMinShift ? s : kMinShift;
}

// 2^s, -126 <= s <= 127.
__device__ __forceinline__ float power2(int s) { return __uint_as_float((s + 127) << 23); }

// Eight codes of a block of exponent s; what is not finite becomes NaN. Codes
// stop at 240 where s is 120: the next, 256, would stand for 2^128.
__device__ __forceinline__ u2 encode8(const float* v, int s) {
  const float scale = power2(-s);
  float t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = v[e] * scale;  // the cast makes NaN of infinities
  if (s == 120) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (__builtin_fabsf(t[e]) > 240.0f && finite(t[e])) t[e] = __builtin_copysignf(240.0f, t[e]);
  }
  u2 q;
  int a = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
  q.x = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], a, true);
  a = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], 0, false);
  q.y = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], a, true);
  return q;
}

__device__ __forceinline__ void decode4(uint32_t q, float scale, float* v) {
  const v2f a = __builtin_amdgcn_cvt_pk_f32_fp8(q, false);
  const v2f b = __builtin_amdgcn_cvt_pk_f32_fp8(q, true);
  v[0] = a.x * scale;
  v[1] = a.y * scale;
  v[2] = b.x * scale;
  v[3] = b.y * scale;
}

__device__ __forceinline__ void decode8(u2 q, float scale, float* v) {
  decode4(q.x, scale, v);
  decode4(q.y, scale, v + 4);
}

}  // namespace garfield
