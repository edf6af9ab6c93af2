// 8-bit checkpoints: making them, from a matrix or its transpose, and giving
// the values back. All are bound by memory: at 8192 x 8192 in bf16 the transposed one takes
// 50 us (4.0 TB/s: lines of 128 bytes of 128 rows), giving back 30 us (6.7 TB/s); 16384 x
// 8192 in bf16 to 8 bits 71 to 79 us (5.7 to 5.1 TB/s).

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
  const int s = block_shift(max16(largest<8>(v)));
  *reinterpret_cast<u2*>(out.values + row * out.ld_values + c) = encode8(v, s);
  if (threadIdx.x % 16 == 0)
    out.exponents[row * out.ld_exponents + b] = static_cast<uint8_t>(s + 127);
}

// The transpose: a workgroup takes 128 rows x 256 bytes of x, the columns of which are
// one block each of the result's rows; neighbouring workgroups read on in the same
// rows. Four lanes to a block, 32 values each, and a lane has as many columns as fit
// a word, which is what it reads from LDS at a time.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_checkpoint_transposed(const T* __restrict__ x,
                                                                  int64_t ld, garfield_block8 out,
                                                                  int64_t blocks, int64_t strips) {
  constexpr int kPer = 4 / sizeof(T), kWords = 64, kCols = kWords * kPer, kVec = 16 / sizeof(T);
  typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  union Piece {
    T t[kVec];
    uint32_t w[4];
  };
  __shared__ uint32_t tile[kBlock8][kWords + 1];
  const int64_t b = blockIdx.x / strips, r0 = b * kBlock8, c0 = blockIdx.x % strips * kCols;
  if (b >= blocks) {
    const int64_t c = c0 + threadIdx.x;
    if (threadIdx.x < kCols && c < out.rows) out.exponents[c * out.ld_exponents + b] = 127;
    return;
  }
#pragma unroll
  for (int i = 0; i < kBlock8 / 16; ++i) {
    const int r = i * 16 + threadIdx.x / 16, c = threadIdx.x % 16 * kVec;
    const int64_t left = r0 + r < out.cols ? out.rows - c0 - c : 0;
    const T* from = x + (r0 + r) * ld + c0 + c;
    Piece p;
    if (left >= kVec) {
      const Vec v = *reinterpret_cast<const Vec*>(from);
#pragma unroll
      for (int e = 0; e < kVec; ++e) p.t[e] = v[e];
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e) p.t[e] = e < left ? from[e] : static_cast<T>(0.0f);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) tile[r][threadIdx.x % 16 * 4 + e] = p.w[e];
  }
  __syncthreads();
  const int word = threadIdx.x / 4, part = threadIdx.x % 4;
  float v[kPer][32];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    union {
      uint32_t w;
      T t[kPer];
    } u;
    u.w = tile[part * 32 + i][word];
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e][i] = static_cast<float>(u.t[e]);
  }
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    float a = largest<32>(v[e]);
    a = __builtin_fmaxf(a, __shfl_xor(a, 1));
    a = __builtin_fmaxf(a, __shfl_xor(a, 2));
    const int64_t row = c0 + word * kPer + e;
    if (row >= out.rows) continue;
    const int s = block_shift(a);
    u4* to = reinterpret_cast<u4*>(out.values + row * out.ld_values + r0 + part * 32);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const u2 lo = encode8(v[e] + 16 * i, s), hi = encode8(v[e] + 16 * i + 8, s);
      u4 q;
      q.x = lo.x;
      q.y = lo.y;
      q.z = hi.x;
      q.w = hi.y;
      to[i] = q;
    }
    if (part == 0) out.exponents[row * out.ld_exponents + b] = static_cast<uint8_t>(s + 127);
  }
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
  const int64_t strips = (out.rows * static_cast<int64_t>(sizeof(T)) + 255) / 256;
  if (transposed)
    launch("checkpoint_transposed", k_checkpoint_transposed<T>,
           dim3(static_cast<uint32_t>(padded * strips)), dim3(kBlock), 0, s, p, ld, out, blocks,
           strips);
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
