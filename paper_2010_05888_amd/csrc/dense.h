// Dense products on the matrix instructions: how operands come from memory to LDS and from
// there to the instruction, for 16- and 32-bit values in both orders.
//
// A tile's operand is a number of columns of the result ("lines") times `depth`, the columns
// that are added up, taken 128 bytes of depth at a time (a block: 64 values, 32 in fp32). An
// operand lies `along` where a line's depth is next to each other in memory, `across` where
// the lines are. LDS holds it as it lies in memory:
//   along: a line's 128 bytes are eight 16-byte pieces, piece c at c ^ (line / 2 % 8);
//   across: a depth's lines are chunks of 16 values, chunk c at c ^ spread(depth).
// The exchanges give the lanes that LDS serves at a time banks of their own. For the 16-bit
// instruction (16 lines, 32 deep) lane l needs line l % 16 and the eight depths from l / 16 * 8
// on: a piece, or two transposing reads of four depths each. For fp32 (4 deep, one value a
// lane) the lane takes the same piece and gives its four values to four instructions, whose
// depths then are in another order, in both operands the same one.
#pragma once

#include <type_traits>

#include "block8.h"
#include "to_lds.h"

namespace garfield {

typedef _Float16 h8v __attribute__((ext_vector_type(8)));

template <typename T>
struct Fragment;
template <>
struct Fragment<__bf16> {
  typedef bf8 type;
};
template <>
struct Fragment<_Float16> {
  typedef h8v type;
};
template <>
struct Fragment<float> {
  typedef v4f type;
};

// A piece's depths added to a 16 x 16 sum, whose rows are a's lines: lane l ends with lines
// l / 16 * 4 to + 3 of a and line l % 16 of b.
__device__ __forceinline__ v4f multiply(bf8 a, bf8 b, v4f sum) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, sum, 0, 0, 0);
}
__device__ __forceinline__ v4f multiply(h8v a, h8v b, v4f sum) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, sum, 0, 0, 0);
}
__device__ __forceinline__ v4f multiply(v4f a, v4f b, v4f sum) {
#pragma unroll
  for (int e = 0; e < 4; ++e) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], sum, 0, 0, 0);
  return sum;
}

typedef __attribute__((address_space(3))) uint8_t* LocalPointer;

// One operand of a tile of LINES lines, brought by WAVES waves.
template <typename T, bool ACROSS, int LINES, int WAVES>
struct Side {
  static constexpr int kSize = sizeof(T), kDepth = 128 / kSize;
  static constexpr int kBytes = LINES * 128;               // of a block in LDS
  static constexpr int kLoads = kBytes / 1024 / WAVES;     // a wave and block
  static constexpr int kRow = ACROSS ? LINES * kSize : 128;  // bytes of a row in LDS
  static constexpr int kRows = 1024 / kRow;                // rows that a load brings
  static_assert(kBytes % (1024 * WAVES) == 0 && kRow <= 1024, "loads are shared out evenly");
  static_assert(ACROSS || 8 * WAVES % 16 == 0, "the exchange is of 16 lines");

  // (16-bit rows of four chunks: two of them are the banks' 256 bytes.)
  static __device__ __forceinline__ int spread(int t) {
    if constexpr (kSize == 4) return t >> 2 & 3;
    else if constexpr (LINES == 64) return (t >> 1 & 1) | (t >> 2 & 2);
    else return (t & 3) | (t >> 1 & 4);
  }

  const char* at;        // of the block that comes next
  int64_t step;          // bytes between blocks
  uint32_t ld;           // bytes between rows
  uint32_t last;         // bytes of the last row that are read
  uint32_t bytes;        // along: of a block, from its first line's to the last line's end
  uint32_t of[kLoads];   // the lane's place in each load
  int deep;              // along: the depth at which the lane's piece starts

  // p: line 0 of the tile at depth 0; `lines` are there. Rows are whole 16-byte pieces, the last
  // one's rest 0, and a block's within 2^30 bytes.
  __device__ __forceinline__ void start(const T* p, int64_t stride, int64_t lines, int wave,
                                        int lane) {
    ld = static_cast<uint32_t>(stride * kSize);
    at = reinterpret_cast<const char*>(p);
    const int row = lane * 16 / kRow, piece = lane % (kRow / 16);
    const int here = lines < LINES ? static_cast<int>(lines) : LINES;
    if constexpr (ACROSS) {
      constexpr int kPieces = kSize;  // of a chunk
      step = kDepth * int64_t{ld};
      last = (here * kSize + 15) / 16 * 16;
      deep = 0;
      bytes = 0;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int t = (i * WAVES + wave) * kRows + row;
        const int chunk = (piece / kPieces) ^ spread(t);
        of[i] = t * ld + (chunk * kPieces + piece % kPieces) * 16;
      }
    } else {
      step = 128;
      last = 128;
      bytes = (here - 1) * ld + (ld < 128 ? ld : 128);  // the next line is not there
      const int chunk = piece ^ ((wave * 8 + row) / 2 % 8);  // that of lines 16 n on too
      deep = chunk * 16 / kSize;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) of[i] = ((i * WAVES + wave) * 8 + row) * ld + chunk * 16;
    }
  }

  // The next block, of which `left` depths are there (none: it reads as 0).
  __device__ __forceinline__ u4 next(int left) {
    uint32_t there = bytes;
    if constexpr (ACROSS)
      there = left <= 0 ? 0 : ((left < kDepth ? left : kDepth) - 1) * ld + last;
    const u4 b = buffer_of(at, there);
    at += step;
    return b;
  }
  // Its load i to LDS at `to`.
  __device__ __forceinline__ void fetch(int i, u4 buffer, int left, int wave, uint32_t to) const {
    // depths past the end are beyond the buffer's
    const uint32_t from = ACROSS || deep < left ? of[i] : 0x7ffffff0u;
    load_to_lds16(buffer, from, to + (i * WAVES + wave) * 1024);
  }

  typedef typename Fragment<T>::type F;
  // The lane's place for the 16 lines from `line` on (a multiple of 16): near(place, i) is that
  // of the i-th 16 lines on, where i is less than a power of two that line / 16 is a multiple of.
  static __device__ __forceinline__ int place(int line, int lane) {
    if constexpr (!ACROSS) {
      const int l = line + lane % 16;
      return l * 128 + ((lane / 16) ^ (l / 2 % 8)) * 16;
    } else if constexpr (kSize == 2) {
      const int t = lane / 16 * 8 + lane % 16 / 4;
      return t * kRow + ((line / 16) ^ spread(t)) * 32 + lane % 4 * 8;
    } else {
      const int t = lane / 16 * 4;
      return t * kRow + ((line / 16) ^ spread(t)) * 64 + lane % 16 * 4;
    }
  }
  static __device__ __forceinline__ int near(int place, int i) {
    return ACROSS ? place ^ (i * 16 * kSize) : place + i * 16 * 128;
  }
  // Half block h of a fragment.
  static __device__ __forceinline__ F read(LocalPointer p, int place, int h) {
    if constexpr (!ACROSS) {
      return *reinterpret_cast<__attribute__((address_space(3))) F*>(p + (h ? place ^ 64 : place));
    } else if constexpr (kSize == 2) {
      typedef __bf16 bf4 __attribute__((ext_vector_type(4)));
      typedef __attribute__((address_space(3))) bf4* At;
      // four and 32 depths on the exchange is the same
      const int first = place + h * 32 * kRow;
      union {
        bf4 half[2];
        F v;
      } t;
      t.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<At>(p + first));
      t.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          reinterpret_cast<At>(p + first + 4 * kRow));
      return t.v;
    } else {
      F v;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[e] = *reinterpret_cast<__attribute__((address_space(3))) float*>(p + place + (h * 16 + e) * kRow);
      return v;
    }
  }
};

}  // namespace garfield
