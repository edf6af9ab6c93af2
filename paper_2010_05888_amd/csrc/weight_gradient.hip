// The weight gradient of a linear layer for each worker: dw = dY^T X over the
// worker's tokens, with X an 8-bit checkpoint. X's values are exact in bf16, so
// the products are bf16 ones with fp32 sums; a dY of more bits is split into
// bf16 parts whose sum it is.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

struct Tokens {
  int64_t first[kWorkersMax + 1];
};

// Part p of v: the leading eight significant bits of what the parts before it
// leave, cut off rather than rounded, so that no part overflows. Parts of what
// is not finite are v itself, then 0.
template <int PARTS>
__device__ __forceinline__ void split(float v, __bf16* part) {
  const bool whole = !finite(v);
  if constexpr (PARTS == 1) {
    part[0] = static_cast<__bf16>(v);
  } else {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
      const float t = __uint_as_float(__float_as_uint(v) & 0xffff0000u);
      part[p] = static_cast<__bf16>(whole ? (p ? 0.0f : v) : t);
      v -= t;
    }
  }
}

template <typename T>
constexpr int parts_of() {
  return sizeof(T) == 4 ? 3 : std::is_same<T, _Float16>::value ? 2 : 1;
}

// A wave takes 16 outputs x 64 inputs of one worker's gradient.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_weight_gradient(const T* __restrict__ dy,
                                                            int64_t outputs, int64_t lddy,
                                                            garfield_block8 x, Tokens tokens,
                                                            float* __restrict__ dw, int64_t ld_dw,
                                                            uint32_t across) {
  constexpr int kParts = parts_of<T>();
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t j0 = (static_cast<int64_t>(blockIdx.x / across) * 4 + wave) * 16;
  const int64_t k0 = static_cast<int64_t>(blockIdx.x % across) * 64;
  if (j0 >= outputs) return;
  const int worker = blockIdx.y;
  const int64_t j = j0 + lane % 16 < outputs ? j0 + lane % 16 : outputs - 1;
  v4f sum[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t end = tokens.first[worker + 1];
  for (int64_t t0 = tokens.first[worker]; t0 < end; t0 += 32) {
    bf8 a[kParts];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int64_t t = t0 + lane / 16 * 8 + e;
      __bf16 part[kParts];
      split<kParts>(t < end ? static_cast<float>(dy[t * lddy + j]) : 0.0f, part);
#pragma unroll
      for (int p = 0; p < kParts; ++p) a[p][e] = part[p];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      int64_t k = k0 + 16 * i + lane % 16;
      k = k < x.cols ? k : x.cols - 1;
      bf8 b;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int64_t t = t0 + lane / 16 * 8 + e;
        float v = 0.0f;
        if (t < end)
          v = __builtin_amdgcn_cvt_f32_fp8(x.values[t * x.ld_values + k], 0) *
              power2(x.exponents[t * x.ld_exponents + k / kBlock8] - 127);
        b[e] = static_cast<__bf16>(v);
      }
#pragma unroll
      for (int p = 0; p < kParts; ++p)
        sum[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[p], b, sum[i], 0, 0, 0);
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int64_t k = k0 + 16 * i + lane % 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int64_t jr = j0 + lane / 16 * 4 + r;
      if (jr < outputs && k < x.cols) dw[worker * ld_dw + jr * x.cols + k] = sum[i][r];
    }
  }
}

template <typename T>
__global__ __launch_bounds__(64) void k_column_sums(const T* __restrict__ dy, int64_t outputs,
                                                    int64_t lddy, Tokens tokens,
                                                    float* __restrict__ dbias, int64_t ld_dbias) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;
  if (j >= outputs) return;
  float sum = 0.0f;
  for (int64_t t = tokens.first[blockIdx.y]; t < tokens.first[blockIdx.y + 1]; ++t)
    sum += static_cast<float>(dy[t * lddy + j]);
  dbias[blockIdx.y * ld_dbias + j] = sum;
}

template <typename T>
void launch_gradient(const WeightGradient& a, const Tokens& tokens, hipStream_t s) {
  const T* dy = static_cast<const T*>(a.dy);
  const uint32_t across = static_cast<uint32_t>((a.x.cols + 63) / 64);
  if (across > 0)
    launch("weight_gradient", k_weight_gradient<T>,
           dim3(across * static_cast<uint32_t>((a.outputs + 63) / 64), a.n), dim3(kBlock), 0, s, dy,
           a.outputs, a.lddy, a.x, tokens, a.dw, a.ld_dw, across);
  if (a.dbias)
    launch("column_sums", k_column_sums<T>, dim3(static_cast<uint32_t>((a.outputs + 63) / 64), a.n),
           dim3(64), 0, s, dy, a.outputs, a.lddy, tokens, a.dbias, a.ld_dbias);
}

}  // namespace

size_t weight_gradient_bytes(int, int64_t, int64_t, int64_t, int64_t, int, const int64_t*) {
  return 0;
}

hipError_t enqueue_weight_gradient(const WeightGradient& a, void*, hipStream_t s) {
  Tokens tokens = {};
  for (int w = 0; w < a.n; ++w) tokens.first[w + 1] = tokens.first[w] + a.counts[w];
  if (a.type == GARFIELD_F32) launch_gradient<float>(a, tokens, s);
  else if (a.type == GARFIELD_BF16) launch_gradient<__bf16>(a, tokens, s);
  else launch_gradient<_Float16>(a, tokens, s);
  return hipGetLastError();
}

}  // namespace garfield
