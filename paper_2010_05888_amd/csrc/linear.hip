// Products of 16- and 32-bit matrices with an epilogue: a linear layer's forward pass, the
// gradient of its input, and of each worker the gradient of its weights.

#include <algorithm>

#include "activation.h"
#include "block8.h"
#include "dense.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

// The epilogue of eight neighbouring outputs of row m; only those below `cols` are touched.
template <typename T>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t m, int64_t j, int64_t cols,
                                       float* v) {
  const int64_t left = cols - j;
  if (left <= 0) return;
  float t[8];
  if (e.before) {
    load8_upto(static_cast<const T*>(e.before) + m * e.ld_before + j, left, t);
    times_slope<8>(e.activation, t, v);
  } else {
    if (e.bias) {
      if (e.bias_f32) load8_upto(static_cast<const float*>(e.bias) + j, left, t);
      else load8_upto(static_cast<const T*>(e.bias) + j, left, t);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += t[i];
    }
    if (e.pre) store8_upto(static_cast<T*>(e.pre) + m * e.ld_pre + j, left, v);
    activate<8>(e.activation, v);
  }
  if (e.residual) {
    load8_upto(static_cast<const T*>(e.residual) + m * e.ld_residual + j, left, t);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += t[i];
  }
  store8_upto(static_cast<T*>(e.out) + m * e.ld_out + j, left, v);
}

// Workgroup id to tile: workgroups go to the eight XCDs in turn, so an XCD's
// share is made contiguous, and inside it eight tiles of rows deep: the tiles that
// an XCD has in work share their rows of both operands in its L2.
// `parts`: shares of the depth, or workers, whose tiles come one part after the other.
struct Place {
  int64_t m, j;
  int part;
};
__device__ __forceinline__ Place place_of(uint32_t id, uint32_t total, uint32_t tiles_m,
                                          uint32_t tiles_j) {
  constexpr uint32_t kXcds = 8, kDeep = 8;
  const uint32_t share = total / kXcds, more = total % kXcds, xcd = id % kXcds;
  uint32_t at = xcd * share + (xcd < more ? xcd : more) + id / kXcds;
  const int part = static_cast<int>(at / (tiles_m * tiles_j));
  at %= tiles_m * tiles_j;
  const uint32_t group = kDeep * tiles_j, first = at / group * kDeep;
  const uint32_t deep = tiles_m - first < kDeep ? tiles_m - first : kDeep;
  return {first + at % group % deep, at % group / deep, part};
}

// A tile's sums: a workgroup of WJ * WM waves makes WM * FB * 16 rows x WJ * FA * 16 columns of
// A B^T, a wave FA x FB products of 16 x 16, block after block. The next block goes from memory
// straight to LDS while the waves work on this one, a few loads at a time between the products.
template <typename T, bool AA, bool BA, int WJ, int WM, int FA, int FB>
struct Tile {
  static constexpr int kWaves = WJ * WM, kCols = WJ * FA * 16, kRows = WM * FB * 16;
  typedef Side<T, AA, kRows, kWaves> SideA;
  typedef Side<T, BA, kCols, kWaves> SideB;
  static constexpr int kStage = SideA::kBytes + SideB::kBytes;
  static constexpr int kLoads = SideA::kLoads + SideB::kLoads;

  // `ones` (with_ones): the sums of A's lines over the depth.
  template <typename Ones>
  static __device__ __forceinline__ void sums(uint8_t* lds, const T* a, int64_t lda, int64_t rows,
                                              const T* b, int64_t ldb, int64_t cols, int64_t depth,
                                              v4f (&sum)[FA][FB], Ones&& ones) {
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wj = wave / WM, wm = wave % WM;
    SideA from_a;
    SideB from_b;
    from_a.start(a, lda, rows, depth, wave, lane);
    from_b.start(b, ldb, cols, depth, wave, lane);
    const uint32_t base = lds_offset(lds);
    constexpr int kDepth = SideA::kDepth;
    const int blocks = static_cast<int>((depth + kDepth - 1) / kDepth);
    auto fetch = [&](int l, int block, int into) {
      const int left = block < blocks ? static_cast<int>(depth - int64_t{block} * kDepth) : 0;
      const uint32_t to = base + into * kStage;
      if (l < SideB::kLoads) from_b.fetch(l, block, left, wave, to + SideA::kBytes);
      else from_a.fetch(l - SideB::kLoads, block, left, wave, to);
    };
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
      for (int k = 0; k < FB; ++k) sum[i][k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    int at_a[FB], at_b[FA];
#pragma unroll
    for (int k = 0; k < FB; ++k) at_a[k] = SideA::place((wm * FB + k) * 16, lane);
#pragma unroll
    for (int i = 0; i < FA; ++i) at_b[i] = SideB::place((wj * FA + i) * 16, lane);
    if (blocks > 0) {
#pragma unroll
      for (int l = 0; l < kLoads; ++l) fetch(l, 0, 0);
    }
    for (int b = 0; b < blocks; ++b) {
      wait_for<0>();
      barrier();  // block b is there, and block b - 1 has been read
      const int next = b + 1, into = next & 1;
      const LocalPointer here_a = (LocalPointer)lds + (b & 1) * kStage;
      const LocalPointer here_b = here_a + SideA::kBytes;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        typename SideA::F af[FB];
        typename SideB::F bf[2];
#pragma unroll
        for (int k = 0; k < FB; ++k) af[k] = SideA::read(here_a, at_a[k], h);
        bf[0] = SideB::read(here_b, at_b[0], h);
        ones(af);
#pragma unroll
        for (int i = 0; i < FA; ++i) {
          if (i + 1 < FA) bf[(i + 1) & 1] = SideB::read(here_b, at_b[i + 1], h);
          if (next < blocks && h == 0) {
#pragma unroll
            for (int l = i * kLoads / FA; l < (i + 1) * kLoads / FA; ++l) fetch(l, next, into);
          }
#pragma unroll
          for (int k = 0; k < FB; ++k) sum[i][k] = multiply(bf[i & 1], af[k], sum[i][k]);
        }
      }
    }
    wait_for<0>();
    barrier();  // LDS is free
  }

  // Every output, eight neighbouring ones of a line at a time: put(line, column, values). A lane
  // has four columns of one line in each of its sums; by way of the wave's own part of LDS,
  // `kPass` sums at a time, they become lines of FA * 16 columns, whose 16-byte piece c lies at
  // c ^ line % kSwap.
  template <typename Put>
  static __device__ __forceinline__ void rows_of(uint8_t* lds, const v4f (&sum)[FA][FB], Put&& put) {
    constexpr int kLine = FA * 64, kRoom = 2 * kStage / kWaves;
    constexpr int kPass = kRoom / (16 * kLine) < FB ? kRoom / (16 * kLine) : FB;
    constexpr int kSwap = FA * 4 < 16 ? FA * 4 : 16, kEights = FA * 2;
    static_assert(kPass > 0 && FB % kPass == 0, "sums go through LDS in equal parts");
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wj = wave / WM, wm = wave % WM;
    uint8_t* const own = lds + wave * kRoom;
#pragma unroll
    for (int k0 = 0; k0 < FB; k0 += kPass) {
#pragma unroll
      for (int k = 0; k < kPass; ++k)
#pragma unroll
        for (int i = 0; i < FA; ++i)
          *reinterpret_cast<v4f*>(own + (k * 16 + lane % 16) * kLine +
                                  ((i * 4 + lane / 16) ^ (lane % kSwap)) * 16) = sum[i][k0 + k];
#pragma unroll 1
      for (int r = lane / kEights; r < kPass * 16; r += 64 / kEights) {
        const int c = lane % kEights * 2;
        v4f v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e)
          v[e] = *reinterpret_cast<const v4f*>(own + r * kLine + ((c + e) ^ (r % kSwap)) * 16);
        float t[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) t[e] = v[e / 4][e % 4];
        put((wm * FB + k0) * 16 + r, wj * FA * 16 + c * 4, t);
      }
    }
  }
};

struct Job {
  const void *a, *b;
  int64_t lda, ldb, rows, cols, depth;
  uint32_t tiles_m, tiles_j;
  int64_t share;   // depths of a share, whole blocks
  float* partial;  // the shares' sums, rows x ld_partial each; null: one share
  int64_t ld_partial;
};

template <typename T, bool AA, bool BA, int WJ, int WM, int FA, int FB>
__global__ __launch_bounds__(64 * WJ * WM) void k_product(Job p, Epilogue to) {
  typedef Tile<T, AA, BA, WJ, WM, FA, FB> Of;
  __shared__ __align__(1024) uint8_t lds[2 * Of::kStage];
  const Place at = place_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_j);
  const int64_t m0 = at.m * Of::kRows, j0 = at.j * Of::kCols, k0 = at.part * p.share;
  const int64_t depth = p.depth - k0 < p.share ? p.depth - k0 : p.share;
  v4f sum[FA][FB];
  Of::sums(lds, static_cast<const T*>(p.a) + (AA ? k0 * p.lda + m0 : m0 * p.lda + k0), p.lda,
           p.rows - m0, static_cast<const T*>(p.b) + (BA ? k0 * p.ldb + j0 : j0 * p.ldb + k0),
           p.ldb, p.cols - j0, depth, sum, [](auto&) {});
  Of::rows_of(lds, sum, [&](int line, int column, float* v) {
    const int64_t m = m0 + line, j = j0 + column;
    if (m >= p.rows) return;
    if (p.partial) {
      float* out = p.partial + (at.part * p.rows + m) * p.ld_partial + j;
      if (j < p.cols) store8_upto(out, p.ld_partial - j, v);
    } else {
      finish<T>(to, m, j, p.cols, v);
    }
  });
}

// The shares' sums added in ascending order, and the epilogue: eight outputs a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_finish(Job p, int shares, Epilogue to) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x;
  const int64_t eights = p.ld_partial / 8;
  if (i >= p.rows * eights) return;
  const int64_t m = i / eights, j = i % eights * 8;
  const float* from = p.partial + m * p.ld_partial + j;
  float sum[8], v[8];
  load8(from, sum);
#pragma unroll 4
  for (int k = 1; k < shares; ++k) {
    load8(from + k * p.rows * p.ld_partial, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
  }
  finish<T>(to, m, j, p.cols, sum);
}

// The workers' tokens, each worker's cut into `splits` shares.
struct Workers {
  int n, splits;
  int64_t first[kWorkersMax + 1];
};

// dw of one worker's share: rows are outputs, columns inputs, the depth its tokens.
template <typename T, int WJ, int WM, int FA, int FB>
__global__ __launch_bounds__(64 * WJ * WM) void k_dense_gradient(Job p, Workers w,
                                                                 float* __restrict__ dw,
                                                                 int64_t ld_dw,
                                                                 float* __restrict__ dbias,
                                                                 int64_t ld_dbias) {
  typedef Tile<T, true, true, WJ, WM, FA, FB> Of;
  __shared__ __align__(1024) uint8_t lds[2 * Of::kStage];
  const Place at = place_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_j);
  const int64_t m0 = at.m * Of::kRows, j0 = at.j * Of::kCols;
  const int worker = at.part % w.n;
  int64_t t0 = w.first[worker], end = w.first[worker + 1];
  constexpr int64_t kDepth = Of::SideA::kDepth;
  const int64_t most = ((end - t0 + kDepth - 1) / kDepth + w.splits - 1) / w.splits * kDepth;
  t0 += at.part / w.n * most;
  end = t0 + most < end ? t0 + most : end;
  const int64_t depth = end > t0 ? end - t0 : 0;
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wj = wave / WM, wm = wave % WM;
  typename Fragment<T>::type one;
#pragma unroll
  for (int e = 0; e < static_cast<int>(16 / sizeof(T)); ++e) one[e] = static_cast<T>(1.0f);
  v4f sum[FA][FB], ones[FB];
#pragma unroll
  for (int k = 0; k < FB; ++k) ones[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  const bool with_bias = dbias && j0 == 0 && wj == 0;
  Of::sums(lds, static_cast<const T*>(p.a) + t0 * p.lda + m0, p.lda, p.rows - m0,
           static_cast<const T*>(p.b) + t0 * p.ldb + j0, p.ldb, p.cols - j0, depth, sum,
           [&](auto& af) {
             if (with_bias) {
#pragma unroll
               for (int k = 0; k < FB; ++k) ones[k] = multiply(one, af[k], ones[k]);
             }
           });
  if (with_bias && lane < 16) {
#pragma unroll
    for (int k = 0; k < FB; ++k) {
      const int64_t m = m0 + (wm * FB + k) * 16 + lane;
      if (m < p.rows) dbias[at.part * ld_dbias + m] = ones[k][0];
    }
  }
  Of::rows_of(lds, sum, [&](int line, int column, float* v) {
    const int64_t m = m0 + line, j = j0 + column;
    if (m < p.rows && j < p.cols)
      store8_upto(dw + at.part * ld_dw + m * p.cols + j, p.cols - j, v);
  });
}

// The splits' gradients added in ascending order: `length` values for each of n workers,
// `next` apart (n * next for each split).
__global__ __launch_bounds__(kBlock) void k_sum_shares(const float* __restrict__ partial,
                                                       int64_t length, int64_t next, int n,
                                                       int splits, float* __restrict__ out,
                                                       int64_t ld) {
  const int64_t i = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 8;
  if (i >= length) return;
  const float* p = partial + blockIdx.y * next + i;
  float sum[8], v[8];
  load8_upto(p, length - i, sum);
#pragma unroll 4
  for (int k = 1; k < splits; ++k) {
    load8_upto(p + k * n * next, length - i, v);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += v[e];
  }
  store8_upto(out + blockIdx.y * ld + i, length - i, sum);
}

// A matrix once more, with rows of whole 16-byte pieces (the last one's rest 0).
template <typename T>
__global__ __launch_bounds__(kBlock) void k_pack_rows(const T* __restrict__ x, int64_t ld,
                                                      int64_t rows, int64_t cols,
                                                      T* __restrict__ out, int64_t ld_out) {
  constexpr int kPiece = 16 / sizeof(T);
  typedef T Piece __attribute__((ext_vector_type(kPiece)));
  typedef T Loose __attribute__((ext_vector_type(kPiece), aligned(sizeof(T))));
  const int64_t pieces = ld_out / kPiece;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < rows * pieces;
       i += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t r = i / pieces, c = i % pieces * kPiece;
    const T* p = x + r * ld + c;
    Piece v;
    if (c + kPiece <= cols) {
      v = *reinterpret_cast<const Loose*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < kPiece; ++e) v[e] = c + e < cols ? p[e] : static_cast<T>(0.0f);
    }
    *reinterpret_cast<Piece*>(out + i * kPiece) = v;
  }
}

// dbias alone, where there are no inputs.
template <typename T>
__global__ __launch_bounds__(64) void k_dense_bias(DenseGradient a, Workers w) {
  const int64_t j = static_cast<int64_t>(blockIdx.x) * 64 + threadIdx.x;
  if (j >= a.outputs) return;
  float sum = 0.0f;
  for (int64_t t = w.first[blockIdx.y]; t < w.first[blockIdx.y + 1]; ++t)
    sum += static_cast<float>(static_cast<const T*>(a.dy)[t * a.lddy + j]);
  a.dbias[blockIdx.y * a.ld_dbias + j] = sum;
}

// Eight values a thread.
template <typename T>
__global__ __launch_bounds__(kBlock) void k_activation_backward(
    const T* __restrict__ dy, int64_t lddy, const T* __restrict__ pre, int64_t ld_pre,
    int activation, T* __restrict__ dp, int64_t lddp, int64_t rows, int64_t cols) {
  const int64_t vectors = (cols + 7) / 8;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x; i < rows * vectors;
       i += static_cast<int64_t>(gridDim.x) * kBlock) {
    const int64_t m = i / vectors, c = i % vectors * 8;
    float g[8], p[8];
    load8_upto(dy + m * lddy + c, cols - c, g);
    load8_upto(pre + m * ld_pre + c, cols - c, p);
    times_slope<8>(activation, p, g);
    store8_upto(dp + m * lddp + c, cols - c, g);
  }
}

constexpr int64_t kMaxApart = int64_t{1} << 27;  // bytes between rows that a load spans

int64_t size_of(int type) { return type == GARFIELD_F32 ? 4 : 2; }
int64_t up_to(int64_t v, int64_t of) { return (v + of - 1) / of * of; }

// Whether the product reads the matrix as it is: whole 16-byte pieces, rows not too far apart.
bool is_whole(const void* p, int64_t ld, int64_t rows, int64_t cols, int64_t size) {
  return reinterpret_cast<uintptr_t>(p) % 16 == 0 && cols * size % 16 == 0 &&
         (rows < 2 || (ld * size % 16 == 0 && ld * size <= kMaxApart));
}

size_t packed_bytes(int64_t rows, int64_t cols, int64_t size) {
  return static_cast<size_t>(up_to(rows * up_to(cols * size, 16), 256));
}

// The matrix as the product reads it; `rest`: the workspace from here on.
template <typename T>
const T* whole(const void* p, int64_t* ld, int64_t rows, int64_t cols, char** rest, hipStream_t s) {
  constexpr int64_t kPiece = 16 / sizeof(T);
  if (is_whole(p, *ld, rows, cols, sizeof(T))) {
    if (rows < 2) *ld = cols;
    return static_cast<const T*>(p);
  }
  T* out = reinterpret_cast<T*>(*rest);
  const int64_t ld_out = up_to(cols, kPiece);
  const int64_t groups = (rows * (ld_out / kPiece) + kBlock - 1) / kBlock, most = int64_t{1} << 23;
  if (groups > 0)
    launch("pack_rows", k_pack_rows<T>, dim3(static_cast<uint32_t>(groups < most ? groups : most)),
           dim3(kBlock), 0, s, static_cast<const T*>(p), *ld, rows, cols, out, ld_out);
  *rest += packed_bytes(rows, cols, sizeof(T));
  *ld = ld_out;
  return out;
}

int64_t tiles_of(int64_t rows, int64_t cols, int size) {
  return ((rows + size - 1) / size) * ((cols + size - 1) / size);
}

// Tiles of 64, 128 or 256 lines, and into how many shares their depth is cut.
struct Plan {
  int size, shares;
  int64_t share;  // depths
};

Plan plan_product(int64_t rows, int64_t cols, int64_t depth, int64_t size) {
  const int64_t block = 128 / size, blocks = (depth + block - 1) / block;
  Plan p = {64, 1, (blocks > 0 ? blocks : 1) * block};
  if (tiles_of(rows, cols, 256) >= 192) {
    p.size = 256;
  } else if (tiles_of(rows, cols, 128) >= 192) {
    p.size = 128;
  } else if (rows > 0 && cols > 0) {
    const int64_t tiles = tiles_of(rows, cols, 64), most = 3 * int64_t{device_cus()};
    const int64_t want = std::min(most / tiles, blocks / 4);
    if (want >= 2) {
      const int64_t per = (blocks + want - 1) / want;
      p.share = per * block;
      p.shares = static_cast<int>((blocks + per - 1) / per);
    }
  }
  return p;
}

template <typename T, bool BA, int WJ, int WM, int FA, int FB>
void launch_tiles(Job p, const Plan& plan, const Epilogue& to, hipStream_t s) {
  p.tiles_m = static_cast<uint32_t>((p.rows + WM * FB * 16 - 1) / (WM * FB * 16));
  p.tiles_j = static_cast<uint32_t>((p.cols + WJ * FA * 16 - 1) / (WJ * FA * 16));
  launch("product", k_product<T, false, BA, WJ, WM, FA, FB>,
         dim3(p.tiles_m * p.tiles_j * plan.shares), dim3(64 * WJ * WM), 0, s, p, to);
}

template <typename T, bool BA>
void choose_product(const Product& of, void* workspace, hipStream_t s) {
  char* rest = static_cast<char*>(workspace);
  Job p = {};
  p.lda = of.a.ld;
  p.ldb = of.b.ld;
  p.a = whole<T>(of.a.p, &p.lda, of.rows, of.depth, &rest, s);
  p.b = BA ? whole<T>(of.b.p, &p.ldb, of.depth, of.cols, &rest, s)
           : whole<T>(of.b.p, &p.ldb, of.cols, of.depth, &rest, s);
  p.rows = of.rows;
  p.cols = of.cols;
  p.depth = of.depth;
  const Plan plan = plan_product(p.rows, p.cols, p.depth, sizeof(T));
  p.share = plan.share;
  if (plan.shares > 1) {
    p.partial = reinterpret_cast<float*>(rest);
    p.ld_partial = up_to(p.cols, 8);
  }
  if (plan.size == 256) launch_tiles<T, BA, 2, 4, 8, 4>(p, plan, of.to, s);
  else if (plan.size == 128) launch_tiles<T, BA, 2, 2, 4, 4>(p, plan, of.to, s);
  else launch_tiles<T, BA, 2, 2, 2, 2>(p, plan, of.to, s);
  if (plan.shares > 1)
    launch("finish", k_finish<T>,
           dim3(static_cast<uint32_t>((p.rows * (p.ld_partial / 8) + kBlock - 1) / kBlock)),
           dim3(kBlock), 0, s, p, plan.shares, of.to);
}

template <typename T>
void launch_product(const Product& p, void* workspace, hipStream_t s) {
  if (p.b.across) choose_product<T, true>(p, workspace, s);
  else choose_product<T, false>(p, workspace, s);
}

// As plan_product, of every worker's gradient: the depth is its tokens.
Plan plan_gradient(const DenseGradient& a, int64_t size) {
  const int64_t block = 128 / size, blocks = (a.tokens / a.n + block - 1) / block;
  Plan p = {64, 1, 0};
  if (tiles_of(a.outputs, a.inputs, 256) * a.n >= 192) p.size = 256;
  else if (tiles_of(a.outputs, a.inputs, 128) * a.n >= 192) p.size = 128;
  else if (a.outputs > 0 && a.inputs > 0) {
    const int64_t tiles = tiles_of(a.outputs, a.inputs, 64) * a.n, most = 3 * int64_t{device_cus()};
    const int64_t want = std::min(most / tiles, blocks / 4);
    if (want >= 2) p.shares = static_cast<int>(std::min<int64_t>(want, 16));
  }
  return p;
}

template <typename T, int WJ, int WM, int FA, int FB>
void launch_gradients(Job p, const Workers& w, float* dw, int64_t ld_dw, float* dbias,
                      int64_t ld_dbias, hipStream_t s) {
  p.tiles_m = static_cast<uint32_t>((p.rows + WM * FB * 16 - 1) / (WM * FB * 16));
  p.tiles_j = static_cast<uint32_t>((p.cols + WJ * FA * 16 - 1) / (WJ * FA * 16));
  // A launch has fewer than 2^32 threads: many workers' tiles take several
  const int64_t tiles = int64_t{p.tiles_m} * p.tiles_j * w.splits;
  const int fit = static_cast<int>(std::min<int64_t>(0xffffffff / (64 * WJ * WM) / tiles, w.n));
  for (int i = 0; i < w.n; i += fit) {
    Workers some = w;
    some.n = w.n - i < fit ? w.n - i : fit;
    for (int k = 0; k <= some.n; ++k) some.first[k] = w.first[i + k];
    launch("dense_gradient", k_dense_gradient<T, WJ, WM, FA, FB>,
           dim3(static_cast<uint32_t>(tiles * some.n)), dim3(64 * WJ * WM), 0, s, p, some,
           dw + i * ld_dw, ld_dw, dbias ? dbias + i * ld_dbias : nullptr, ld_dbias);
  }
}

template <typename T>
void launch_gradient(const DenseGradient& a, void* workspace, hipStream_t s) {
  Workers w = {};
  w.n = a.n;
  for (int i = 0; i < a.n; ++i) w.first[i + 1] = w.first[i] + a.counts[i];
  if (a.inputs == 0) {
    if (a.dbias)
      launch("dense_bias", k_dense_bias<T>, dim3(static_cast<uint32_t>((a.outputs + 63) / 64), a.n),
             dim3(64), 0, s, a, w);
    return;
  }
  const Plan plan = plan_gradient(a, sizeof(T));
  w.splits = plan.shares;
  char* rest = static_cast<char*>(workspace);
  Job p = {};
  p.lda = a.lddy;
  p.ldb = a.ldx;
  p.a = whole<T>(a.dy, &p.lda, a.tokens, a.outputs, &rest, s);
  p.b = whole<T>(a.x, &p.ldb, a.tokens, a.inputs, &rest, s);
  p.rows = a.outputs;
  p.cols = a.inputs;
  float *dw = a.dw, *dbias = a.dbias;
  int64_t ld_dw = a.ld_dw, ld_dbias = a.ld_dbias;
  const int64_t length = a.outputs * a.inputs;
  if (plan.shares > 1) {
    dw = reinterpret_cast<float*>(rest);
    ld_dw = up_to(length, 4);
    if (dbias) dbias = dw + plan.shares * a.n * ld_dw;
    ld_dbias = a.outputs;
  }
  if (plan.size == 256) launch_gradients<T, 2, 4, 8, 4>(p, w, dw, ld_dw, dbias, ld_dbias, s);
  else if (plan.size == 128) launch_gradients<T, 2, 2, 4, 4>(p, w, dw, ld_dw, dbias, ld_dbias, s);
  else launch_gradients<T, 2, 2, 2, 2>(p, w, dw, ld_dw, dbias, ld_dbias, s);
  if (plan.shares > 1) {
    auto add = [&](const float* from, int64_t n, int64_t next, float* out, int64_t ld) {
      launch("sum_shares", k_sum_shares,
             dim3(static_cast<uint32_t>((n + 8 * kBlock - 1) / (8 * kBlock)), a.n), dim3(kBlock), 0,
             s, from, n, next, a.n, plan.shares, out, ld);
    };
    add(dw, length, ld_dw, a.dw, a.ld_dw);
    if (a.dbias) add(dbias, a.outputs, a.outputs, a.dbias, a.ld_dbias);
  }
}

}  // namespace

size_t product_bytes(const Product& p) {
  const int64_t size = size_of(p.type);
  size_t bytes = 0;
  if (!is_whole(p.a.p, p.a.ld, p.rows, p.depth, size)) bytes += packed_bytes(p.rows, p.depth, size);
  const int64_t rows = p.b.across ? p.depth : p.cols, cols = p.b.across ? p.cols : p.depth;
  if (!is_whole(p.b.p, p.b.ld, rows, cols, size)) bytes += packed_bytes(rows, cols, size);
  const Plan plan = plan_product(p.rows, p.cols, p.depth, size);
  if (plan.shares > 1) bytes += static_cast<size_t>(plan.shares) * p.rows * up_to(p.cols, 8) * 4;
  return bytes;
}

hipError_t enqueue_product(const Product& p, void* workspace, hipStream_t s) {
  if (p.type == GARFIELD_F32) launch_product<float>(p, workspace, s);
  else if (p.type == GARFIELD_BF16) launch_product<__bf16>(p, workspace, s);
  else launch_product<_Float16>(p, workspace, s);
  return hipGetLastError();
}

size_t dense_gradient_bytes(const DenseGradient& a) {
  if (a.outputs == 0 || a.inputs == 0) return 0;
  const int64_t size = size_of(a.type);
  size_t bytes = 0;
  if (!is_whole(a.dy, a.lddy, a.tokens, a.outputs, size))
    bytes += packed_bytes(a.tokens, a.outputs, size);
  if (!is_whole(a.x, a.ldx, a.tokens, a.inputs, size)) bytes += packed_bytes(a.tokens, a.inputs, size);
  const Plan plan = plan_gradient(a, size);
  if (plan.shares > 1)
    bytes += static_cast<size_t>(plan.shares) * a.n *
             (up_to(a.outputs * a.inputs, 4) + a.outputs) * sizeof(float);
  return bytes;
}

hipError_t enqueue_dense_gradient(const DenseGradient& a, void* workspace, hipStream_t s) {
  if (a.type == GARFIELD_F32) launch_gradient<float>(a, workspace, s);
  else if (a.type == GARFIELD_BF16) launch_gradient<__bf16>(a, workspace, s);
  else launch_gradient<_Float16>(a, workspace, s);
  return hipGetLastError();
}

template <typename T>
static void launch_slope(const void* dy, int64_t lddy, const void* pre, int64_t ld_pre,
                         int activation, void* dp, int64_t lddp, int64_t rows, int64_t cols,
                         hipStream_t s) {
  const int64_t groups = (rows * ((cols + 7) / 8) + kBlock - 1) / kBlock, most = int64_t{1} << 23;
  launch("activation_backward", k_activation_backward<T>,
         dim3(static_cast<uint32_t>(groups < most ? groups : most)), dim3(kBlock), 0, s,
         static_cast<const T*>(dy), lddy, static_cast<const T*>(pre), ld_pre, activation,
         static_cast<T*>(dp), lddp, rows, cols);
}

hipError_t enqueue_activation_backward(const void* dy, int64_t lddy, const void* pre,
                                       int64_t ld_pre, int activation, void* dp, int64_t lddp,
                                       int type, int64_t rows, int64_t cols, hipStream_t s) {
  if (type == GARFIELD_F32)
    launch_slope<float>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  else if (type == GARFIELD_BF16)
    launch_slope<__bf16>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  else
    launch_slope<_Float16>(dy, lddy, pre, ld_pre, activation, dp, lddp, rows, cols, s);
  return hipGetLastError();
}

}  // namespace garfield
