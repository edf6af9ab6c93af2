// The product of 8-bit blocks, out = X W^T + bias.
//
// Fast: the scaled matrix instruction makes 16 x 16 outputs from 128 columns,
// each row's 128 codes with one exponent. A block is 128 codes with one
// exponent, so the instruction takes both as they are stored and nothing is left
// to scale. Its adder keeps 14 bits: with one product of 2^8 among the eight that
// it adds together, another of 2^-5 is kept and one of 2^-6 lost (products of
// normal values: 1.2e-5 of the result's size off, 7e-5 with wider spreads).
// Otherwise: codes times 2^s are exact in bf16, and four bf16 instructions of half
// the rate add the same products with fp32 sums.
//
// W is the instructions' first operand (its rows are the result's rows), so a
// lane ends with four neighbouring outputs of one token. Lane l gives row
// l % 16 and 32 of the 128 columns, the same ones for both operands.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

__device__ __forceinline__ i8v load32(const uint8_t* p) {
  union {
    u4 h[2];
    i8v v;
  } t;
  t.h[0] = reinterpret_cast<const u4*>(p)[0];
  t.h[1] = reinterpret_cast<const u4*>(p)[1];
  return t.v;
}

// Eight codes of a lane as bf16 values.
__device__ __forceinline__ bf8 decode_bf16(uint32_t lo, uint32_t hi, float scale) {
  typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
  union {
    bf2 h[4];
    bf8 v;
  } t;
  t.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  t.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  t.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  t.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return t.v;
}

// c + a b over a block; sa and sb are the exponents as they are stored.
template <bool FAST>
__device__ __forceinline__ v4f product(i8v a, i8v b, v4f c, int sa, int sb) {
  if constexpr (FAST) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, sa, 0, sb);
  } else {
    const float fa = power2(sa - 127), fb = power2(sb - 127);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(decode_bf16(a[2 * i], a[2 * i + 1], fa),
                                                  decode_bf16(b[2 * i], b[2 * i + 1], fb), c, 0, 0,
                                                  0);
    return c;
  }
}

// Four outputs of one token (fewer at the row's end).
template <typename T>
__device__ __forceinline__ void store_outputs(T* out, const float* bias, int64_t j, int64_t outputs,
                                              v4f v) {
  typedef T Four __attribute__((ext_vector_type(4), aligned(sizeof(T))));
  if (j + 4 <= outputs) {
    Four t;
#pragma unroll
    for (int e = 0; e < 4; ++e) t[e] = static_cast<T>(bias ? v[e] + bias[j + e] : v[e]);
    *reinterpret_cast<Four*>(out + j) = t;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < outputs) out[j + e] = static_cast<T>(bias ? v[e] + bias[j + e] : v[e]);
  }
}

// A wave takes 16 outputs of 64 tokens, operands straight from memory.
template <typename T, bool FAST>
__global__ __launch_bounds__(kBlock) void k_linear8(garfield_block8 x, garfield_block8 w,
                                                    const float* __restrict__ bias, T* out,
                                                    int64_t ld, uint32_t across) {
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t j0 = (static_cast<int64_t>(blockIdx.x % across) * 4 + wave) * 16;
  const int64_t m0 = static_cast<int64_t>(blockIdx.x / across) * 64;
  if (j0 >= w.rows) return;
  const int64_t j = j0 + lane % 16 < w.rows ? j0 + lane % 16 : w.rows - 1;
  const uint8_t* wv = w.values + j * w.ld_values + lane / 16 * 32;
  const uint8_t* we = w.exponents + j * w.ld_exponents;
  const uint8_t *xv[4], *xe[4];
  v4f sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int64_t m = m0 + 16 * i + lane % 16;
    m = m < x.rows ? m : x.rows - 1;
    xv[i] = x.values + m * x.ld_values + lane / 16 * 32;
    xe[i] = x.exponents + m * x.ld_exponents;
    sum[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
  const int64_t blocks = (x.cols + kBlock8 - 1) / kBlock8;
  for (int64_t b = 0; b < blocks; ++b) {
    const i8v a = load32(wv + b * kBlock8);
    const int sa = we[b];
#pragma unroll
    for (int i = 0; i < 4; ++i) sum[i] = product<FAST>(a, load32(xv[i] + b * kBlock8), sum[i], sa, xe[i][b]);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t m = m0 + 16 * i + lane % 16;
    if (m < x.rows) store_outputs(out + m * ld, bias, j0 + lane / 16 * 4, w.rows, sum[i]);
  }
}

template <typename T, bool FAST>
void launch_linear8(const garfield_block8& x, const garfield_block8& w, const float* bias,
                    void* out, int64_t ld, hipStream_t s) {
  const uint32_t across = static_cast<uint32_t>((w.rows + 63) / 64);
  launch("linear8", k_linear8<T, FAST>, dim3(across * static_cast<uint32_t>((x.rows + 63) / 64)),
         dim3(kBlock), 0, s, x, w, bias, static_cast<T*>(out), ld, across);
}

template <typename T>
void choose_linear8(const garfield_block8& x, const garfield_block8& w, const float* bias,
                    bool fast, void* out, int64_t ld, hipStream_t s) {
  if (fast) launch_linear8<T, true>(x, w, bias, out, ld, s);
  else launch_linear8<T, false>(x, w, bias, out, ld, s);
}

}  // namespace

size_t linear8_bytes(int64_t, int64_t, int64_t) { return 0; }

hipError_t enqueue_linear8(const garfield_block8& x, const garfield_block8& w, const float* bias,
                           bool fast, void* out, int type, int64_t ld, void*, hipStream_t s) {
  if (type == GARFIELD_F32) choose_linear8<float>(x, w, bias, fast, out, ld, s);
  else if (type == GARFIELD_BF16) choose_linear8<__bf16>(x, w, bias, fast, out, ld, s);
  else choose_linear8<_Float16>(x, w, bias, fast, out, ld, s);
  return hipGetLastError();
}

}  // namespace garfield
