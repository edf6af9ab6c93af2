// The weight gradient of a linear layer for each worker: dw = dY^T X over the
// worker's tokens, with X an 8-bit checkpoint. X's values are exact in bf16, so
// the products are bf16 ones with fp32 sums; a dY of more bits is split into
// bf16 parts whose sum it is, one after the other in the same sum.
//
// Both operands have the tokens, over which the sum runs, as rows: LDS holds them
// as they lie in memory and transposing reads give the matrix instruction its
// columns. A wave's part of dw is 128 inputs wide, one block of X with one exponent
// a token: X's codes become bf16 in LDS once for all the waves; dY goes straight
// there.
//
// Bounds: the matrix cores' bf16 rate for many tokens a worker (one worker's 16384 x
// 4096 x 4096: 490 us, 1120 TFLOP/s), the stores of dw, 4 bytes for 2 * tokens operations,
// for few (19 workers without tokens: 229 us, 5.6 TB/s); 19 workers' 16384 tokens take 690 to
// 740 us, nearly their sum.

#include <type_traits>

#include "block8.h"
#include "internal.h"
#include "timing.h"
#include "to_lds.h"
#include "worker.h"

namespace garfield {

namespace {

typedef __bf16 bf4 __attribute__((ext_vector_type(4)));

// The workers' tokens, each worker's cut into `splits` shares of whole steps.
struct Tokens {
  int64_t first[kWorkersMax + 1];
  int n, splits;
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

// dY as k_weight_gradient reads it (5.3 us for 1000 x 1001 in fp32): its parts, one
// matrix after the other, rows of a multiple of eight columns (the last ones 0).
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

// (Rows of four chunks: two of them are the banks' 256 bytes.)
template <int CHUNKS>
__device__ __forceinline__ int spread(int t) {
  return CHUNKS == 4 ? (t >> 1 & 1) | (t >> 2 & 2) : (t & 3) | (t >> 1 & 4);
}

// Four values of a column for each lane's column: 16 lanes read 4 rows of 16
// neighbouring columns, lane l from row l / 4 and column l % 4 * 4 on, and lane l
// gets column l's.
typedef __attribute__((address_space(3))) uint8_t* LocalBytes;
__device__ __forceinline__ bf4 read_column(LocalBytes p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
      reinterpret_cast<__attribute__((address_space(3))) bf4*>(p));
}

__device__ __forceinline__ bf8 join(bf4 a, bf4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A workgroup makes 64 * FB outputs x 128 * WK inputs of one worker's gradient, a
// wave 16 * FB x 128 of them, step after step of 32 tokens. In step s, step s + 3
// starts on its way to LDS; between the products every thread turns its 16 codes of
// step s + 2 into bf16; and the first operands of step s + 1, which the last step's
// barrier has made good, are read before this one's. So dY has four places, X's
// codes two, its values three.
// Rows are 32-byte chunks of 16 values, and 32 lanes read a chunk of tokens t to
// t + 3 and t + 8 to t + 11 at a time: chunk c of token t lies at c ^ spread(t), which
// gives each its own eighth of the banks.
// Tokens past the share's last read as 0 in both operands.
// A worker's splits are gradients of their own, ld_dw apart like the workers' (and
// the workers of a split n * ld_dw): k_sum_splits adds them.
template <int WK, int FB>
__global__ __launch_bounds__(256 * WK, 2) void k_weight_gradient(
    Parts a, garfield_block8 x, Tokens tokens, float* __restrict__ dw, int64_t ld_dw,
    float* __restrict__ dbias, int64_t ld_dbias, int64_t outputs, uint32_t tiles_j,
    uint32_t tiles_k, bool whole_lines) {
  constexpr int kFA = 8, kWaves = 4 * WK, kTileJ = 64 * FB, kTileK = 128 * WK;
  constexpr int kRowJ = kTileJ * 2, kRowK = kTileK * 2;  // bytes
  constexpr int kY = kTokens * kRowJ, kX = kTokens * kRowK, kCodes = kTokens * kTileK;
  constexpr int kExponents = 256 * kWaves;  // a word a thread
  constexpr int kAtX = 4 * kY, kAtCodes = kAtX + 3 * kX, kAtExponents = kAtCodes + 2 * kCodes;
  constexpr int kFetchRows = 1024 / kRowJ;  // rows that a wave's load brings
  constexpr int kLoads = FB / WK;           // of dY, a wave and step
  constexpr int kFetches = kLoads + 2;
  static_assert(FB % WK == 0, "loads are shared out evenly");
  __shared__ __align__(1024) uint8_t lds[kAtExponents + 2 * kExponents];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wj = wave % 4, wk = wave / 4;

  // An XCD's share of the tiles is contiguous (workgroups go to the XCDs in turn), and
  // eight tiles of outputs deep: the 32 that it has in work share their columns of dY and
  // X in its L2 (8 x 16 + 4 x 8 KB a step, where 32 x 1 would be 520 KB).
  const uint32_t total = gridDim.x, share = total / 8, more = total % 8, xcd = blockIdx.x % 8;
  uint32_t at = xcd * share + (xcd < more ? xcd : more) + blockIdx.x / 8;
  const int share_of = at / (tiles_j * tiles_k);  // worker by worker in every split
  const int worker = share_of % tokens.n;
  at %= tiles_j * tiles_k;
  constexpr uint32_t kDeep = 8;
  const uint32_t group = kDeep * tiles_k, deep0 = at / group * kDeep;
  const uint32_t deep = tiles_j - deep0 < kDeep ? tiles_j - deep0 : kDeep;
  const int64_t j0 = static_cast<int64_t>(deep0 + at % group % deep) * kTileJ;
  const int block0 = at % group / deep * WK;
  int64_t first = tokens.first[worker], end = tokens.first[worker + 1];
  const int64_t all = (end - first + kTokens - 1) / kTokens;
  const int64_t most = (all + tokens.splits - 1) / tokens.splits * kTokens;
  first += share_of / tokens.n * most;
  end = first + most < end ? first + most : end;
  first = first < end ? first : end;
  const int64_t per_part = (end - first + kTokens - 1) / kTokens, steps = per_part * a.parts;

  // the lane's places in a step of dY, X and X's exponents
  uint32_t from[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int t = (i * kWaves + wave) * kFetchRows + lane * 16 / kRowJ;
    const int piece = lane % (kRowJ / 16);
    const int column = (((piece / 2) ^ spread<4 * FB>(t)) * 2 + piece % 2) * 8;
    from[i] = (static_cast<uint32_t>(t) * static_cast<uint32_t>(a.ld) + column) * 2;
  }
  const int xt = threadIdx.x / (8 * WK), xp = threadIdx.x % (8 * WK);  // a token's 16 codes
  const uint32_t from_x = static_cast<uint32_t>(xt) * static_cast<uint32_t>(x.ld_values) + xp * 16;
  const uint32_t from_e =
      static_cast<uint32_t>(xt) * static_cast<uint32_t>(x.ld_exponents) + xp / 8;
  const uint32_t base = lds_offset(lds);

  // What the next fetch reads. The bounds of a part's last step end its rows at the
  // worker's last token; X's end at its last block, for a tile may reach beyond.
  const int blocks = static_cast<int>((x.cols + kBlock8 - 1) / kBlock8);
  const int here = blocks - block0 < WK ? blocks - block0 : WK;
  const uint32_t rows_before =
      static_cast<uint32_t>(end - first - (per_part - 1) * kTokens) - 1;  // the last one
  const uint32_t last_y = (rows_before * static_cast<uint32_t>(a.ld) +
                           static_cast<uint32_t>(a.columns - j0)) * 2;
  const uint32_t last_x = rows_before * static_cast<uint32_t>(x.ld_values) + here * kBlock8;
  const uint32_t last_e = rows_before * static_cast<uint32_t>(x.ld_exponents) + here;
  const uint32_t full_y = ((kTokens - 1) * static_cast<uint32_t>(a.ld) +
                           static_cast<uint32_t>(a.columns - j0)) * 2;
  const uint32_t full_x =
      (kTokens - 1) * static_cast<uint32_t>(x.ld_values) + here * kBlock8;
  const uint32_t full_e = (kTokens - 1) * static_cast<uint32_t>(x.ld_exponents) + here;
  const __bf16* at_y = a.dy + first * a.ld + j0;
  const uint8_t* at_x = x.values + first * x.ld_values + static_cast<int64_t>(block0) * kBlock8;
  const uint8_t* at_e = x.exponents + first * x.ld_exponents + block0;
  int64_t left = per_part, parts_left = steps > 0 ? a.parts : 0;
  // A step's loads, in four parts: dY, X, and its exponents with what the next step needs.
  auto fetch_part = [&](int part, int place, int odd) {
    const bool last = left == 1, none = parts_left <= 0;  // fetches go past the end
    if (part < 2) {
      const u4 of_y = buffer_of(at_y, none ? 0 : last ? last_y : full_y);
#pragma unroll
      for (int i = part * kLoads / 2; i < (part + 1) * kLoads / 2; ++i)
        load_to_lds16(of_y, from[i], base + place * kY + (i * kWaves + wave) * 1024);
    } else if (part == 2) {
      const u4 of_x = buffer_of(at_x, none ? 0 : last ? last_x : full_x);
      load_to_lds16(of_x, from_x, base + kAtCodes + odd * kCodes + wave * 1024);
    } else {
      const u4 of_e = buffer_of(at_e, none ? 0 : last ? last_e : full_e);
      load_to_lds1(of_e, from_e, base + kAtExponents + odd * kExponents + wave * 256);
      at_y += kTokens * a.ld;
      at_x += kTokens * x.ld_values;
      at_e += kTokens * x.ld_exponents;
      if (--left == 0) {
        left = per_part;
        --parts_left;
        at_y += a.next - per_part * kTokens * a.ld;
        at_x -= per_part * kTokens * x.ld_values;
        at_e -= per_part * kTokens * x.ld_exponents;
      }
    }
  };
  auto fetch = [&](int place, int odd) {
#pragma unroll
    for (int part = 0; part < 4; ++part) fetch_part(part, place, odd);
  };
  // the thread's own codes, as its wave has fetched them
  struct Codes {
    u4 code;
    uint32_t exponent;
  };
  auto read_codes = [&](int odd) {
    return Codes{
        *reinterpret_cast<const u4*>(lds + kAtCodes + odd * kCodes + threadIdx.x * 16),
        *reinterpret_cast<const uint32_t*>(lds + kAtExponents + odd * kExponents + threadIdx.x * 4)};
  };
  const int to_x = xt * kRowK + (xp ^ spread<8>(xt)) * 32;
  auto decode = [&](Codes c, int place) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    union {
      bf2 h[8];
      u4 v[2];
    } t;
    const float scale = __uint_as_float(c.exponent << 23);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      t.h[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.code[i], scale, false);
      t.h[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c.code[i], scale, true);
    }
    u4* to = reinterpret_cast<u4*>(lds + kAtX + place * kX + to_x);
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
  const bool with_bias = dbias && block0 == 0 && wk == 0;

  // lane's places in a step: token 8 (l / 16) + l % 16 / 4, and four tokens on
  const int t0 = lane / 16 * 8 + lane % 16 / 4, in_chunk = lane % 4 * 8;
  const LocalBytes local = (LocalBytes)lds;
  LocalBytes near_y[FB], next_y[FB], near_x[kFA], next_x[kFA];
#pragma unroll
  for (int k = 0; k < FB; ++k) {
    const int c = wj * FB + k;
    near_y[k] = local + t0 * kRowJ + (c ^ spread<4 * FB>(t0)) * 32 + in_chunk;
    next_y[k] = local + (t0 + 4) * kRowJ + (c ^ spread<4 * FB>(t0 + 4)) * 32 + in_chunk;
  }
#pragma unroll
  for (int i = 0; i < kFA; ++i) {
    const int c = wk * kFA + i;
    near_x[i] = local + kAtX + t0 * kRowK + (c ^ spread<8>(t0)) * 32 + in_chunk;
    next_x[i] = local + kAtX + (t0 + 4) * kRowK + (c ^ spread<8>(t0 + 4)) * 32 + in_chunk;
  }

  bf8 y[FB], xf[kFA];
  auto read_y = [&](int place) {
#pragma unroll
    for (int k = 0; k < FB; ++k)
      y[k] = join(read_column(near_y[k] + place * kY), read_column(next_y[k] + place * kY));
  };
  auto read_x = [&](int i, int place) {
    xf[i] = join(read_column(near_x[i] + place * kX), read_column(next_x[i] + place * kX));
  };
  auto multiply = [&](int i) {
#pragma unroll
    for (int k = 0; k < FB; ++k)
      sum[i][k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf[i], y[k], sum[i][k], 0, 0, 0);
  };
  if (steps > 0) {
    fetch(0, 0);
    fetch(1, 1);
    wait_for<0>();
    decode(read_codes(0), 0);
    decode(read_codes(1), 1);
    wait_for_lds();
    fetch(2, 0);
    barrier();
    read_y(0);
    read_x(0, 0);
    read_x(1, 0);
    int of_x = 0;  // X's place of step s
    for (int64_t s = 0; s < steps; ++s) {
      const int of_y = s & 3, odd = s & 1;
      const int next_x = of_x == 2 ? 0 : of_x + 1, after_x = next_x == 2 ? 0 : next_x + 1;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        read_x(i + 2, of_x);
        fetch_part(i, (of_y + 3) & 3, 1 - odd);
        multiply(i);
      }
      wait_for<kFetches>();  // step s + 2 is there
      const Codes codes = read_codes(odd);
      read_x(6, of_x);
      read_x(7, of_x);
      multiply(4);
      multiply(5);
      decode(codes, after_x);
      multiply(6);
      multiply(7);
      if (with_bias) {
#pragma unroll
        for (int k = 0; k < FB; ++k)
          ones[k] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one, y[k], ones[k], 0, 0, 0);
      }
      wait_for_lds();
      read_y((s + 1) & 3);
      read_x(0, next_x);
      read_x(1, next_x);
      barrier_alone();
      of_x = next_x;
    }
  }
  wait_for<0>();  // the last loads, which bring zeros
  barrier();      // LDS is free

  // A lane has four neighbouring inputs of one output, 16 outputs a wave; by way of the
  // wave's part of LDS they become whole rows of 128 inputs, 32 lanes each.
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  constexpr int kRow = 128 * 4 + 16;  // bytes; the rest spreads rows over the banks
  static_assert(kWaves * 16 * kRow <= sizeof(lds), "the waves' parts fit");
  uint8_t* const own = lds + wave * 16 * kRow;
  const int64_t k0 = static_cast<int64_t>(block0 + wk) * kBlock8 + lane % 32 * 4;
  const int64_t left_k = x.cols - k0;
  // Whole lines go past the caches (19 workers, 2048 x 4096 x 4096: 267 us, and 310 by way of
  // them; with 16384 tokens 686 and 671); parts of lines stay for their other parts (11
  // workers, 500 x 2001 x 1999: 68 us, and 72 past them).
  auto store = [&](auto past_caches) {
#pragma unroll
    for (int k = 0; k < FB; ++k) {
      const int64_t j = j0 + (wj * FB + k) * 16;
      if (with_bias && lane < 16 && j + lane < outputs)
        dbias[share_of * ld_dbias + j + lane] = ones[k][0];
#pragma unroll
      for (int i = 0; i < kFA; ++i)
        *reinterpret_cast<v4f*>(own + lane % 16 * kRow + i * 64 + lane / 16 * 16) = sum[i][k];
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const int row = r + lane / 32;
        const v4f t = *reinterpret_cast<const v4f*>(own + row * kRow + lane % 32 * 16);
        if (j + row >= outputs) continue;
        float* to = dw + share_of * ld_dw + (j + row) * x.cols + k0;
        if (left_k >= 4) {
          Four v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = t[e];
          if constexpr (decltype(past_caches)::value)
            __builtin_nontemporal_store(v, reinterpret_cast<Four*>(to));
          else
            *reinterpret_cast<Four*>(to) = v;
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (e < left_k) to[e] = t[e];
        }
      }
    }
  };
  if (whole_lines) store(std::true_type());
  else store(std::false_type());
}

// The splits' gradients added in ascending order: sums of `length` values for each of
// n workers, `next` values apart in partial (n * next for each split). A pass over
// memory; its bytes are part of plan_gradient's choice.
__global__ __launch_bounds__(kBlock) void k_sum_splits(const float* __restrict__ partial,
                                                       int64_t length, int64_t next, int n,
                                                       int splits, float* __restrict__ out,
                                                       int64_t ld) {
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 4;
  if (i >= length) return;
  const float* p = partial + blockIdx.y * next + i;
  float* to = out + blockIdx.y * ld + i;
  if (i + 4 <= length) {
    Four sum = *reinterpret_cast<const Four*>(p);
#pragma unroll 4
    for (int k = 1; k < splits; ++k) sum += *reinterpret_cast<const Four*>(p + k * n * next);
    *reinterpret_cast<Four*>(to) = sum;
  } else {
    for (int e = 0; i + e < length; ++e) {
      float sum = p[e];
      for (int k = 1; k < splits; ++k) sum += p[k * n * next + e];
      to[e] = sum;
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
  const size_t bytes =
      static_cast<size_t>(parts_of_type(type)) * tokens * ((outputs + 7) / 8 * 8) * 2;
  return (bytes + 255) / 256 * 256;
}

// How a call is tiled: 64 * fb outputs x 128 * wk inputs, and into how many shares a
// worker's tokens are cut.
struct Plan {
  int wk, fb, splits;
};

// A round of workgroups costs about their time alone on a CU, which for a step of 32
// tokens is, in units of the largest tile's: 256 x 256, one a CU, 1; two of 128 x 128 on
// a CU 0.72; three of 64 x 128 0.68 (a round of 512 steps on one card: 487 us, 371 and, two
// thirds full, 320). Few tiles of many tokens leave CUs idle: their tokens are cut
// into up to 16 shares of at least eight steps, whose sums cost a pass over splits * 4
// bytes for each value of dw (as long as some 8 steps): one worker's 16384 x 2048 x 4096
// takes 270 us so, and 458, 371 or 572 us uncut in the three forms.
Plan plan_gradient(int parts, int64_t tokens, int64_t outputs, int64_t inputs, int n) {
  struct Shape {
    int wk, fb, slots;
    double time;
  };
  static constexpr Shape kShapes[] = {{2, 4, 1, 1.0}, {1, 2, 2, 0.72}, {1, 1, 3, 0.68}};
  const int cus = device_cus();
  const double steps = static_cast<double>((tokens / n + kTokens) / kTokens) * parts;
  Plan best = {1, 1, 1};
  double least = 1e300;
  for (const Shape& f : kShapes) {
    const int64_t tiles = ((outputs + 64 * f.fb - 1) / (64 * f.fb)) *
                          ((inputs + 128 * f.wk - 1) / (128 * f.wk)) * n;
    for (int splits = 1; splits <= 16; splits *= 2) {
      if (splits > 1 && (steps < 8.0 * splits || splits * tiles > 4 * f.slots * cus)) break;
      const int64_t slots = static_cast<int64_t>(f.slots) * cus;
      const double rounds = static_cast<double>((tiles * splits + slots - 1) / slots);
      const double sums = splits > 1 ? 8.0 + splits : 0.0;
      const double time = rounds * f.time * (steps / splits + 4.0) + sums;
      if (time < least) {
        least = time;
        best = {f.wk, f.fb, splits};
      }
    }
  }
  return best;
}

template <int WK, int FB>
void launch_gradient(const Parts& p, const WeightGradient& a, const Tokens& tokens, float* dw,
                     int64_t ld_dw, float* dbias, int64_t ld_dbias, hipStream_t s) {
  const uint32_t tiles_j = static_cast<uint32_t>((a.outputs + 64 * FB - 1) / (64 * FB));
  const uint32_t tiles_k = static_cast<uint32_t>((a.x.cols + 128 * WK - 1) / (128 * WK));
  // whether tiles' rows are whole lines of 128 bytes
  const bool whole_lines = reinterpret_cast<uintptr_t>(dw) % 128 == 0 && ld_dw % 32 == 0 &&
                           a.x.cols % 32 == 0;
  // A launch has fewer than 2^32 threads. Few outputs of many inputs and workers have more
  // tiles (one worker's always fit, and tokens in shares are few tiles' only): the workers
  // then take several launches.
  const int64_t tiles = int64_t{tiles_j} * tiles_k * tokens.splits;
  const int fit = static_cast<int>(0xffffffff / (256 * WK) / tiles);
  for (int w = 0; w < tokens.n; w += fit) {
    Tokens some = tokens;
    some.n = tokens.n - w < fit ? tokens.n - w : fit;
    for (int i = 0; i <= some.n; ++i) some.first[i] = tokens.first[w + i];
    launch("weight_gradient", k_weight_gradient<WK, FB>,
           dim3(static_cast<uint32_t>(tiles * some.n)), dim3(256 * WK), 0, s, p, a.x, some,
           dw + w * ld_dw, ld_dw, dbias ? dbias + w * ld_dbias : nullptr, ld_dbias, a.outputs,
           tiles_j, tiles_k, whole_lines);
  }
}

void launch_sums(const float* partial, int64_t length, int64_t next, const Tokens& tokens,
                 float* out, int64_t ld, hipStream_t s) {
  launch("sum_splits", k_sum_splits,
         dim3(static_cast<uint32_t>((length + 4 * kBlock - 1) / (4 * kBlock)), tokens.n),
         dim3(kBlock), 0, s, partial, length, next, tokens.n, tokens.splits, out, ld);
}

template <typename T>
void choose_gradient(const WeightGradient& a, Tokens& tokens, void* workspace, hipStream_t s) {
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
  char* rest = static_cast<char*>(workspace);
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
    rest += packed_bytes(a.type, a.tokens, a.outputs);
  } else {
    p.dy = static_cast<const __bf16*>(a.dy);
    p.columns = a.outputs;
    p.ld = a.lddy;
  }
  const Plan plan = plan_gradient(p.parts, a.tokens, a.outputs, a.x.cols, a.n);
  tokens.splits = plan.splits;
  const int64_t length = a.outputs * a.x.cols;
  float *dw = a.dw, *dbias = a.dbias;
  int64_t ld_dw = a.ld_dw, ld_dbias = a.ld_dbias;
  if (plan.splits > 1) {
    dw = reinterpret_cast<float*>(rest);
    ld_dw = (length + 3) / 4 * 4;
    if (dbias) dbias = dw + plan.splits * a.n * ld_dw;
    ld_dbias = a.outputs;
  }
  if (plan.wk == 2) launch_gradient<2, 4>(p, a, tokens, dw, ld_dw, dbias, ld_dbias, s);
  else if (plan.fb == 2) launch_gradient<1, 2>(p, a, tokens, dw, ld_dw, dbias, ld_dbias, s);
  else launch_gradient<1, 1>(p, a, tokens, dw, ld_dw, dbias, ld_dbias, s);
  if (plan.splits > 1) {
    launch_sums(dw, length, ld_dw, tokens, a.dw, a.ld_dw, s);
    if (a.dbias) launch_sums(dbias, a.outputs, a.outputs, tokens, a.dbias, a.ld_dbias, s);
  }
}

}  // namespace

size_t weight_gradient_bytes(int type, int64_t tokens, int64_t outputs, int64_t inputs,
                             const void* dy, int64_t lddy, int n, const int64_t*) {
  if (inputs == 0 || outputs == 0) return 0;
  const size_t packed =
      packs(type, outputs, lddy, dy) ? packed_bytes(type, tokens, outputs) : 0;
  const Plan plan = plan_gradient(parts_of_type(type), tokens, outputs, inputs, n);
  const size_t gradient = static_cast<size_t>((outputs * inputs + 3) / 4 * 4 + outputs);
  return packed + (plan.splits > 1 ? plan.splits * n * gradient * sizeof(float) : 0);
}

hipError_t enqueue_weight_gradient(const WeightGradient& a, void* workspace, hipStream_t s) {
  Tokens tokens = {};
  tokens.n = a.n;
  tokens.splits = 1;
  for (int w = 0; w < a.n; ++w) tokens.first[w + 1] = tokens.first[w] + a.counts[w];
  if (a.type == GARFIELD_F32) choose_gradient<float>(a, tokens, workspace, s);
  else if (a.type == GARFIELD_BF16) choose_gradient<__bf16>(a, tokens, workspace, s);
  else choose_gradient<_Float16>(a, tokens, workspace, s);
  return hipGetLastError();
}

}  // namespace garfield
