// The weight gradient of a linear layer for each worker: dw = dY^T X over the
// worker's tokens, with X an 8-bit checkpoint. X's values are exact in bf16, so
// the products are bf16 ones with fp32 sums; a dY of more bits is split into
// bf16 parts whose sum it is, one after the other in the same sum.
//
// Both operands have the tokens, over which the sum runs, as rows: LDS holds them
// as they lie in memory and transposing reads give the matrix instruction its
// columns. A tile of dw takes 128 inputs, so one block of X and one exponent a
// token: X goes through registers, where its codes become bf16 once for all the
// waves; dY goes straight to LDS. Two workgroups share a CU, so that one's
// products cover the other's stores: dw is 4 bytes for 2 tokens operations.

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "to_lds.h"
#include "worker.h"

namespace garfield {

namespace {

typedef __bf16 bf4 __attribute__((ext_vector_type(4)));

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
int parts_of_type(int type) { return type == GARFIELD_F32 ? 3 : type == GARFIELD_F16 ? 2 : 1; }

// dY as k_weight_gradient reads it: its parts, one matrix after the other, rows
// of a multiple of eight columns (the last ones 0).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_pack(const T* __restrict__ dy, int64_t tokens,
                                                 int64_t outputs, int64_t lddy, int64_t vectors,
                                                 __bf16* __restrict__ packed) {
  constexpr int kParts = parts_of<T>();
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  if (i >= tokens * vectors) return;
  const int64_t t = i / vectors, c = i % vectors * 8;
  float v[8];
  load8_upto(dy + t * lddy + c, outputs - c, v);
  bf8 part[kParts];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    __bf16 p[kParts];
    split<kParts>(v[e], p);
#pragma unroll
    for (int k = 0; k < kParts; ++k) part[k][e] = p[k];
  }
#pragma unroll
  for (int k = 0; k < kParts; ++k)
    *reinterpret_cast<bf8*>(packed + ((k * tokens + t) * vectors * 8 + c)) = part[k];
}

// What k_weight_gradient takes for dY: `parts` matrices of bf16, rows 16-byte
// aligned, columns a multiple of eight, 32 rows within 32 bits.
struct Parts {
  const __bf16* dy;
  int64_t columns, ld, next;  // elements between rows, and between parts
  int parts;
};

constexpr int kTokens = 32;  // a step's: the matrix instruction's depth

// Four values of a column for each lane's column: 16 lanes read 4 rows of 16
// neighbouring columns, lane l from row l / 4 and column l % 4 * 4 on, and lane l
// gets column l's.
__device__ __forceinline__ bf4 read_column(const uint8_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      (__attribute__((address_space(3))) bf4*)(LocalPtr)p);
}

__device__ __forceinline__ bf8 join(bf4 a, bf4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A workgroup makes 64 * FB outputs x 128 inputs of one worker's gradient, a wave
// 16 * FB of the outputs, step after step of 32 tokens. While step s is
// multiplied, step s + 2 is on its way to LDS; then every thread turns its 16 codes
// of step s + 1 into bf16. So dY has three places, X's codes two, its values two.
// Rows of 32-byte chunks (16 values), chunk c of token t at c ^ (t % 8) (t % 4 where
// a row has four): the four rows that 16 lanes read lie in different banks.
// Tokens past the worker's last read as 0 in both operands.
template <int FB>
__global__ __launch_bounds__(256, 2) void k_weight_gradient(Parts a, garfield_block8 x,
                                                            Tokens tokens, float* __restrict__ dw,
                                                            int64_t ld_dw,
                                                            float* __restrict__ dbias,
                                                            int64_t ld_dbias, int64_t outputs,
                                                            uint32_t tiles_j, uint32_t tiles_k) {
  constexpr int kFA = 8, kTileJ = 64 * FB, kTileK = 128;
  constexpr int kRowJ = kTileJ * 2, kRowK = kTileK * 2;  // bytes
  constexpr int kY = kTokens * kRowJ, kX = kTokens * kRowK, kCodes = kTokens * kTileK;
  constexpr int kExponents = 4 * 256;  // a word a thread
  constexpr int kAtX = 3 * kY, kAtCodes = kAtX + 2 * kX, kAtExponents = kAtCodes + 2 * kCodes;
  constexpr int kMaskJ = FB == 1 ? 3 : 7;
  constexpr int kFetchRows = 1024 / kRowJ;  // rows that a wave's load brings
  constexpr int kFetches = FB + 2;          // a step's loads of a wave
  __shared__ __align__(1024) uint8_t lds[kAtExponents + 2 * kExponents];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;

  // an XCD's share of the tiles is contiguous (workgroups go to the XCDs in turn)
  const uint32_t total = gridDim.x, share = total / 8, more = total % 8, xcd = blockIdx.x % 8;
  uint32_t at = xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const int worker = at / (tiles_j * tiles_k);
  at %= tiles_j * tiles_k;
  const int64_t j0 = static_cast<int64_t>(at % tiles_j) * kTileJ;
  const int block = at / tiles_j;
  const int64_t first = tokens.first[worker], end = tokens.first[worker + 1];
  const int64_t steps = (end - first + kTokens - 1) / kTokens * a.parts;

  // the lane's places in a step of dY, X and X's exponents
  uint32_t from[FB];
#pragma unroll
  for (int i = 0; i < FB; ++i) {
    const int t = (i * 4 + wave) * kFetchRows + lane * 16 / kRowJ;
    const int piece = lane % (kRowJ / 16);
    const int column = (((piece / 2) ^ (t & kMaskJ)) * 2 + piece % 2) * 8;
    from[i] = (static_cast<uint32_t>(t) * static_cast<uint32_t>(a.ld) + column) * 2;
  }
  const int xt = threadIdx.x / 8, xp = threadIdx.x % 8;  // eight threads to a token
  const uint32_t from_x = static_cast<uint32_t>(xt) * static_cast<uint32_t>(x.ld_values) + xp * 16;
  const uint32_t from_e = static_cast<uint32_t>(xt) * static_cast<uint32_t>(x.ld_exponents);
  const uint32_t base = lds_offset(lds);

  int64_t fetch_t = first, fetched = 0;  // the step to be fetched
  const __bf16* part = a.dy;
  auto fetch = [&](int place) {
    const int64_t left = end - fetch_t;
    const uint32_t rows =
        fetched >= steps ? 0 : static_cast<uint32_t>(left < kTokens ? left : kTokens);
    const uint32_t beyond = rows ? rows - 1 : 0;  // rows before the last
    const u4 of_y = buffer_of(part + fetch_t * a.ld + j0,
                              rows ? (beyond * static_cast<uint32_t>(a.ld) +
                                      static_cast<uint32_t>(a.columns - j0)) * 2
                                   : 0);
    const u4 of_x = buffer_of(x.values + fetch_t * x.ld_values + block * kTileK,
                              rows ? beyond * static_cast<uint32_t>(x.ld_values) + kTileK : 0);
    const u4 of_e = buffer_of(x.exponents + fetch_t * x.ld_exponents + block,
                              rows ? beyond * static_cast<uint32_t>(x.ld_exponents) + 1 : 0);
#pragma unroll
    for (int i = 0; i < FB; ++i)
      load_to_lds16(of_y, from[i], base + place * kY + (i * 4 + wave) * 1024);
    const int odd = fetched & 1;
    load_to_lds16(of_x, from_x, base + kAtCodes + odd * kCodes + wave * 1024);
    load_to_lds1(of_e, from_e, base + kAtExponents + odd * kExponents + wave * 256);
    ++fetched;
    fetch_t += kTokens;
    if (fetch_t >= end) {
      fetch_t = first;
      part += a.next;
    }
  };
  // the thread's own codes, as its wave has fetched them
  auto decode = [&](int odd) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    union {
      bf2 h[8];
      u4 v[2];
    } t;
    const u4 code = *reinterpret_cast<const u4*>(lds + kAtCodes + odd * kCodes + threadIdx.x * 16);
    const uint32_t e = *reinterpret_cast<const uint32_t*>(lds + kAtExponents + odd * kExponents +
                                                          threadIdx.x * 4);
    const float scale = __uint_as_float(e << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[i], scale, false);
      t.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code[i], scale, true);
    }
    u4* to = reinterpret_cast<u4*>(lds + kAtX + odd * kX + xt * kRowK + ((xp ^ (xt & 7)) * 32));
    to[0] = t.v[0];
    to[1] = t.v[1];
  };

  v4f sum[kFA][FB], ones[FB];
#pragma unroll
  for (int k = 0; k < FB; ++k) {
    ones[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < kFA; ++i) sum[i][k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  }
  bf8 one;
#pragma unroll
  for (int e = 0; e < 8; ++e) one[e] = static_cast<__bf16>(1.0f);
  const bool with_bias = dbias && block == 0;

  // lane's places in a step: token 8 (l / 16) + l % 16 / 4, and four tokens on
  const int t0 = lane / 16 * 8 + lane % 16 / 4, in_chunk = lane % 4 * 8;
  const int near_j = t0 * kRowJ + (t0 & kMaskJ) * 32 + in_chunk;
  const int next_j = (t0 + 4) * kRowJ + ((t0 + 4) & kMaskJ) * 32 + in_chunk;
  const int near_k = t0 * kRowK + (t0 & 7) * 32 + in_chunk;
  const int next_k = (t0 + 4) * kRowK + ((t0 + 4) & 7) * 32 + in_chunk;

  if (steps > 0) {
    fetch(0);
    fetch(1);
    wait_for<kFetches>();
    decode(0);
    barrier();
  }
  int place = 0;
  for (int64_t s = 0; s < steps; ++s) {
    const int next = place == 2 ? 0 : place + 1;
    fetch(next == 2 ? 0 : next + 1);
    const uint8_t* py = lds + place * kY;
    const uint8_t* px = lds + kAtX + (s & 1) * kX;
    bf8 y[FB];
#pragma unroll
    for (int k = 0; k < FB; ++k) {
      const int c = (wave * FB + k) * 32;
      y[k] = join(read_column(py + (near_j ^ c)), read_column(py + (next_j ^ c)));
    }
#pragma unroll
    for (int i = 0; i < kFA; ++i) {
      const bf8 xf =
          join(read_column(px + (near_k ^ (i * 32))), read_column(px + (next_k ^ (i * 32))));
#pragma unroll
      for (int k = 0; k < FB; ++k)
        sum[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, y[k], sum[i][k], 0, 0, 0);
    }
    if (with_bias) {
#pragma unroll
      for (int k = 0; k < FB; ++k)
        ones[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, y[k], ones[k], 0, 0, 0);
    }
    wait_for<kFetches>();  // step s + 1 is there
    decode((s + 1) & 1);
    barrier();
    place = next;
  }
  wait_for<0>();  // the last loads bring zeros to LDS that is free again after this

  // a lane has four neighbouring inputs of one output
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  const int64_t k0 = static_cast<int64_t>(block) * kTileK + lane / 16 * 4;
#pragma unroll
  for (int k = 0; k < FB; ++k) {
    const int64_t j = j0 + (wave * FB + k) * 16 + lane % 16;
    if (j >= outputs) continue;
    if (with_bias && lane < 16) dbias[worker * ld_dbias + j] = ones[k][0];
    float* row = dw + worker * ld_dw + j * x.cols + k0;
#pragma unroll
    for (int i = 0; i < kFA; ++i) {
      if (k0 + i * 16 + 4 <= x.cols) {
        Four t;
#pragma unroll
        for (int e = 0; e < 4; ++e) t[e] = sum[i][k][e];
        *reinterpret_cast<Four*>(row + i * 16) = t;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (k0 + i * 16 + e < x.cols) row[i * 16 + e] = sum[i][k][e];
      }
    }
  }
}

// dbias alone, where there are no inputs.
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

bool packs(int type, int64_t outputs, int64_t lddy, const void* dy) {
  return type != GARFIELD_BF16 || outputs % 8 || lddy % 8 || lddy > (int64_t{1} << 24) ||
         reinterpret_cast<uintptr_t>(dy) % 16;
}

size_t packed_bytes(int type, int64_t tokens, int64_t outputs) {
  return static_cast<size_t>(parts_of_type(type)) * tokens * ((outputs + 7) / 8 * 8) * 2;
}

template <int FB>
void launch_gradient(const Parts& p, const WeightGradient& a, const Tokens& tokens, hipStream_t s) {
  const uint32_t tiles_j = static_cast<uint32_t>((a.outputs + 64 * FB - 1) / (64 * FB));
  const uint32_t tiles_k = static_cast<uint32_t>((a.x.cols + kBlock8 - 1) / kBlock8);
  launch("weight_gradient", k_weight_gradient<FB>, dim3(tiles_j * tiles_k * a.n), dim3(256), 0, s,
         p, a.x, tokens, a.dw, a.ld_dw, a.dbias, a.ld_dbias, a.outputs, tiles_j, tiles_k);
}

template <typename T>
void choose_gradient(const WeightGradient& a, const Tokens& tokens, void* workspace,
                     hipStream_t s) {
  const T* dy = static_cast<const T*>(a.dy);
  if (a.x.cols == 0) {
    if (a.dbias)
      launch("column_sums", k_column_sums<T>,
             dim3(static_cast<uint32_t>((a.outputs + 63) / 64), a.n), dim3(64), 0, s, dy,
             a.outputs, a.lddy, tokens, a.dbias, a.ld_dbias);
    return;
  }
  Parts p = {};
  p.parts = parts_of<T>();
  if (packs(a.type, a.outputs, a.lddy, a.dy)) {
    const int64_t vectors = (a.outputs + 7) / 8;
    __bf16* packed = static_cast<__bf16*>(workspace);
    if (a.tokens > 0)
      launch("pack", k_pack<T>,
             dim3(static_cast<uint32_t>((a.tokens * vectors + kBlock - 1) / kBlock)), dim3(kBlock),
             0, s, dy, a.tokens, a.outputs, a.lddy, vectors, packed);
    p.dy = packed;
    p.columns = p.ld = vectors * 8;
    p.next = a.tokens * p.ld;
  } else {
    p.dy = static_cast<const __bf16*>(a.dy);
    p.columns = a.outputs;
    p.ld = a.lddy;
  }
  const int64_t tiles_k = (a.x.cols + kBlock8 - 1) / kBlock8 * a.n;
  if ((a.outputs + 255) / 256 * tiles_k >= 512) launch_gradient<4>(p, a, tokens, s);
  else if ((a.outputs + 127) / 128 * tiles_k >= 512) launch_gradient<2>(p, a, tokens, s);
  else launch_gradient<1>(p, a, tokens, s);
}

}  // namespace

size_t weight_gradient_bytes(int type, int64_t tokens, int64_t outputs, int64_t inputs,
                             const void* dy, int64_t lddy, int, const int64_t*) {
  return inputs > 0 && packs(type, outputs, lddy, dy) ? packed_bytes(type, tokens, outputs) : 0;
}

hipError_t enqueue_weight_gradient(const WeightGradient& a, void* workspace, hipStream_t s) {
  Tokens tokens = {};
  for (int w = 0; w < a.n; ++w) tokens.first[w + 1] = tokens.first[w] + a.counts[w];
  if (a.type == GARFIELD_F32) choose_gradient<float>(a, tokens, workspace, s);
  else if (a.type == GARFIELD_BF16) choose_gradient<__bf16>(a, tokens, workspace, s);
  else choose_gradient<_Float16>(a, tokens, workspace, s);
  return hipGetLastError();
}

}  // namespace garfield
