// 8-bit checkpoints: making them, from a matrix or its transpose, and giving
// the values back.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

int64_t blocks_of(int64_t cols) { return (cols + kBlock8 - 1) / kBlock8; }
int64_t padded_blocks(int64_t cols) { return (blocks_of(cols) + 3) / 4 * 4; }

// Sixteen lanes to a block, eight values to a lane.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint(const T* __restrict__ x, int64_t ld,
                                                       garfield_block8 out, int64_t blocks,
                                                       int64_t padded) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * (kBlock / 16) + threadIdx.x / 16;
  if (i >= out.rows * padded) return;
  const int64_t row = i / padded, b = i % padded;
  if (b >= blocks) {
    if (threadIdx.x % 16 == 0) out.exponents[row * out.ld_exponents + b] = 127;
    return;
  }
  const int64_t c = b * kBlock8 + threadIdx.x % 16 * 8;
  float v[8];
  load8_upto(x + row * ld + c, out.cols - c, v);
  float a = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) a = __builtin_fmaxf(a, magnitude(v[e]));
  const int s = block_shift(max16(a));
  *reinterpret_cast<u2*>(out.values + row * out.ld_values + c) = encode8(v, s);
  if (threadIdx.x % 16 == 0)
    out.exponents[row * out.ld_exponents + b] = static_cast<uint8_t>(s + 127);
}

// The transpose: a workgroup takes 128 rows x 64 columns of x, which are one
// block of each of 64 rows of the result. Four lanes to a block, 32 values each.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint_transposed(const T* __restrict__ x,
                                                                  int64_t ld, garfield_block8 out,
                                                                  int64_t blocks, int64_t padded) {
  __shared__ float tile[kBlock8][65];
  const int64_t b = blockIdx.x % padded, r0 = b * kBlock8, c0 = blockIdx.x / padded * 64;
  if (b >= blocks) {
    const int64_t c = c0 + threadIdx.x;
    if (threadIdx.x < 64 && c < out.rows) out.exponents[c * out.ld_exponents + b] = 127;
    return;
  }
  for (int r = threadIdx.x / 8; r < kBlock8; r += kBlock / 8) {
    const int c = threadIdx.x % 8 * 8;
    float v[8] = {};
    if (r0 + r < out.cols && c0 + c < out.rows)
      load8_upto(x + (r0 + r) * ld + c0 + c, out.rows - c0 - c, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) tile[r][c + e] = v[e];
  }
  __syncthreads();
  const int col = threadIdx.x / 4, part = threadIdx.x % 4;
  float v[32];
  float a = 0.0f;
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    v[i] = tile[part * 32 + i][col];
    a = __builtin_fmaxf(a, magnitude(v[i]));
  }
  a = __builtin_fmaxf(a, __shfl_xor(a, 1));
  a = __builtin_fmaxf(a, __shfl_xor(a, 2));
  if (c0 + col >= out.rows) return;
  const int s = block_shift(a);
  u4* to = reinterpret_cast<u4*>(out.values + (c0 + col) * out.ld_values + r0 + part * 32);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const u2 lo = encode8(v + 16 * i, s), hi = encode8(v + 16 * i + 8, s);
    u4 q;
    q.x = lo.x;
    q.y = lo.y;
    q.z = hi.x;
    q.w = hi.y;
    to[i] = q;
  }
  if (part == 0) out.exponents[(c0 + col) * out.ld_exponents + b] = static_cast<uint8_t>(s + 127);
}

template <typename T>
__global__ __launch_bounds__(kBlock) void k_restore(garfield_block8 in, T* __restrict__ out,
                                                    int64_t ld, int64_t vectors) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= in.rows * vectors) return;
  const int64_t row = i / vectors, c = i % vectors * 8;
  const int s = in.exponents[row * in.ld_exponents + c / kBlock8] - 127;
  float v[8];
  decode8(*reinterpret_cast<const u2*>(in.values + row * in.ld_values + c), power2(s), v);
  store8_upto(out + row * ld + c, in.cols - c, v);
}

template <typename T>
void launch_checkpoint(const void* x, int64_t ld, bool transposed, const garfield_block8& out,
                       hipStream_t s) {
  const T* p = static_cast<const T*>(x);
  const int64_t blocks = blocks_of(out.cols), padded = padded_blocks(out.cols);
  if (transposed)
    launch("checkpoint_transposed", k_checkpoint_transposed<T>,
           dim3(static_cast<uint32_t>(padded * ((out.rows + 63) / 64))), dim3(kBlock), 0, s, p, ld,
           out, blocks, padded);
  else
    launch("checkpoint", k_checkpoint<T>,
           dim3(static_cast<uint32_t>((out.rows * padded + kBlock / 16 - 1) / (kBlock / 16))),
           dim3(kBlock), 0, s, p, ld, out, blocks, padded);
}

template <typename T>
void launch_restore(const garfield_block8& c, void* out, int64_t ld, hipStream_t s) {
  const int64_t vectors = (c.cols + 7) / 8;
  launch("restore", k_restore<T>,
         dim3(static_cast<uint32_t>((c.rows * vectors + kBlock - 1) / kBlock)), dim3(kBlock), 0, s,
         c, static_cast<T*>(out), ld, vectors);
}

}  // namespace

hipError_t enqueue_checkpoint(const void* x, int type, int64_t rows, int64_t cols, int64_t ld,
                              bool transposed, const garfield_block8& out, hipStream_t s) {
  if (type == GARFIELD_F32) launch_checkpoint<float>(x, ld, transposed, out, s);
  else if (type == GARFIELD_BF16) launch_checkpoint<__bf16>(x, ld, transposed, out, s);
  else launch_checkpoint<_Float16>(x, ld, transposed, out, s);
  return hipGetLastError();
}

hipError_t enqueue_restore(const garfield_block8& c, void* out, int type, int64_t ld,
                           hipStream_t s) {
  if (type == GARFIELD_F32) launch_restore<float>(c, out, ld, s);
  else if (type == GARFIELD_BF16) launch_restore<__bf16>(c, out, ld, s);
  else launch_restore<_Float16>(c, out, ld, s);
  return hipGetLastError();
}

}  // namespace garfield
