// Products of 16- and 32-bit matrices with an epilogue: a linear layer's forward pass, the
// gradient of its input, and of each worker the gradient of its weights.
//
// All three are A B^T with the depth along or across each operand (dense.h), in one kernel's
// three forms: X W^T, dY W with W across, and dY^T X with both across and a worker's tokens as
// its depth. Products are those of the values as they are, sums fp32: fp32 on its own matrix
// instruction, at a sixteenth of the 16-bit ones' rate.
//
// Bounds: the matrix cores' rate, and power (8192^3 in bf16: 800 to 860 us, 1280 to 1370 TFLOP/s; in
// fp32 7500 to 7800 us, 141 to 147 TFLOP/s of 157), and then what an epilogue reads, computes and
// writes, which no products hide: 16384 x 8192 x 2048 takes 465 to 485 us, with gelu and p 540 to
// 570, back through gelu 540 to 580, of which 268 MB more at a copy's rate are 51. (Passes with
// pauses; without, power holds a card back by up to 15% more. A comment's pairs are of one run.)
// For one token B's bytes, for small sizes latency.

#include <algorithm>
#include <type_traits>

#include "activation.h"
#include "block8.h"
#include "dense.h"
#include "internal.h"
#include "timing.h"
#include "worker.h"

namespace garfield {

namespace {

// The epilogue of N neighbouring outputs of row m, all of them there. What it reads of other
// matrices is asked for ahead of the sums.
template <typename T, int N>
struct Finish {
  typedef T Raw __attribute__((ext_vector_type(N), aligned(sizeof(T))));
  Raw before, residual;

  static __device__ __forceinline__ Raw raw(const void* p, int64_t at) {
    return *reinterpret_cast<const Raw*>(static_cast<const T*>(p) + at);
  }
  static __device__ __forceinline__ void store(const Epilogue& e, void* p, int64_t at,
                                               const float* v) {
    Raw t;
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = static_cast<T>(v[i]);
    Raw* const to = reinterpret_cast<Raw*>(static_cast<T*>(p) + at);
    if (e.past_caches) __builtin_nontemporal_store(t, to);
    else *to = t;
  }

  __device__ __forceinline__ void ask(const Epilogue& e, int64_t m, int64_t j) {
    if (e.before) before = raw(e.before, m * e.ld_before + j);
    if (e.residual) residual = raw(e.residual, m * e.ld_residual + j);
  }

  __device__ __forceinline__ void put(const Epilogue& e, int64_t m, int64_t j, float* v) const {
    if (e.before) {
      float t[N];
#pragma unroll
      for (int i = 0; i < N; ++i) t[i] = static_cast<float>(before[i]);
      times_slope<N>(e.activation, t, v);
    } else {
      if (e.bias) {
        typedef float Bias __attribute__((ext_vector_type(N), aligned(4)));
        if (e.bias_f32) {
          const Bias t = *reinterpret_cast<const Bias*>(static_cast<const float*>(e.bias) + j);
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] += t[i];
        } else {
          const Raw t = raw(e.bias, j);
#pragma unroll
          for (int i = 0; i < N; ++i) v[i] += static_cast<float>(t[i]);
        }
      }
      if (e.pre) store(e, e.pre, m * e.ld_pre + j, v);
      activate<N>(e.activation, v);
    }
    if (e.residual) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] += static_cast<float>(residual[i]);
    }
    store(e, e.out, m * e.ld_out + j, v);
  }

  // What is there of eight outputs, one after the other.
  template <typename Value>
  static __device__ __forceinline__ void some(const Epilogue& e, int64_t m, int64_t j,
                                              int64_t left, Value&& value) {
#pragma unroll 1
    for (int i = 0; i < left; ++i) {
      Finish<T, 1> one;
      float x = value(i);
      one.ask(e, m, j + i);
      one.put(e, m, j + i, &x);
    }
  }
};

// Workgroup id to tile: workgroups go to the eight XCDs in turn, so an XCD's
// share is made contiguous, and inside it four tiles of rows deep: the tiles that
// an XCD has in work share their rows of both operands in its L2, and write next to each
// other (eight deep, 16384 x 8192 x 2048 takes 484 us, so 465; weight gradients below).
// `parts`: shares of the depth, or workers, whose tiles come one part after the other.
struct Place {
  int64_t m, j;
  int part;
};
__device__ __forceinline__ Place place_of(uint32_t id, uint32_t total, uint32_t tiles_m,
                                          uint32_t tiles_j) {
  constexpr uint32_t kXcds = 8, kDeep = 4;
  const uint32_t share = total / kXcds, more = total % kXcds, xcd = id % kXcds;
  uint32_t at = xcd * share + (xcd < more ? xcd : more) + id / kXcds;
  const int part = static_cast<int>(at / (tiles_m * tiles_j));
  at %= tiles_m * tiles_j;
  const uint32_t group = kDeep * tiles_j, first = at / group * kDeep;
  const uint32_t deep = tiles_m - first < kDeep ? tiles_m - first : kDeep;
  return {first + at % group % deep, at % group / deep, part};
}

// What a tile is made of: line 0 of both operands at depth 0, the lines and depths that are there.
template <typename T>
struct Parts {
  const T *a, *b;
  int64_t rows, cols, depth;
};

// A tile of WM * FB * 16 rows x WJ * FA * 16 columns of A B^T by a workgroup of WJ * WM waves: a
// wave has FA x FB products of 16 x 16, block after block, in two halves. While it multiplies
// one half it reads the next one's operands, so that nothing but the one barrier of a block, in
// its middle, is waited for: there the block has been read, and the one after the next starts on
// its way to its place, a load between every few products, straight to LDS.
// 8192^3 in bf16: 800 to 860 us (a library's product 700 to 790), of zeros 650 to 700 (530 to 580): power
// bounds both; the matrix cores are busy 74% of the time, what they wait for are the loads' issue
// (100 us) and the barrier (50). LDS is read 29% of the time and no bank is waited for. What was
// slower: waves of 128 x 128, one a SIMD (1220); a block's loads all in its first products (815);
// one workgroup for many tiles, the next one's first block on its way during the epilogue (564
// against 535 us for 16384 x 8192 x 2048 with gelu and p: its loads wait for its stores; a new
// workgroup's do not).
template <typename T, bool AA, bool BA, int WJ, int WM, int FA, int FB>
struct Tile {
  static constexpr int kWaves = WJ * WM, kCols = WJ * FA * 16, kRows = WM * FB * 16;
  typedef Side<T, AA, kRows, kWaves> SideA;
  typedef Side<T, BA, kCols, kWaves> SideB;
  static constexpr int kStage = SideA::kBytes + SideB::kBytes;
  static constexpr int kLoads = SideA::kLoads + SideB::kLoads;
  static constexpr int kDepth = SideA::kDepth;
  // Blocks in LDS or on their way. Three of small tiles in 16 bits: 512 x 4096 x 4096 takes 29 us so
  // and 33 in two, other sizes up to 4% less or more; fp32 tiles, which wait for their products,
  // are 3 to 5% slower in three, weight gradients 2%.
  static constexpr int kStages = sizeof(T) == 2 && !AA && kRows * kCols <= 64 * 64 ? 3 : 2;
  static constexpr int kLds = kStages * kStage;

  // also(af): what else is done with A's fragments.
  template <typename Also>
  static __device__ __forceinline__ void sums(uint8_t* lds, int64_t lda, int64_t ldb,
                                              const Parts<T>& p, v4f (&sum)[FA][FB], Also&& also) {
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int wj = wave / WM, wm = wave % WM;
    SideA from_a;
    SideB from_b;
    from_a.start(p.a, lda, p.rows, wave, lane);
    from_b.start(p.b, ldb, p.cols, wave, lane);
    const uint32_t base = lds_offset(lds);
    const uint32_t blocks = static_cast<uint32_t>((p.depth + kDepth - 1) / kDepth);
    int left = static_cast<int>(p.depth);  // depths from the next block on
    u4 of_a, of_b;
    auto next = [&] {
      of_a = from_a.next(left);
      of_b = from_b.next(left);
    };
    auto fetch = [&](int l, int into) {
      const uint32_t to = base + into * kStage;
      if (l < SideB::kLoads) from_b.fetch(l, of_b, left, wave, to + SideA::kBytes);
      else from_a.fetch(l - SideB::kLoads, of_a, left, wave, to);
    };
    const int at_a = SideA::place(wm * FB * 16, lane), at_b = SideB::place(wj * FA * 16, lane);
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
      for (int k = 0; k < FB; ++k) sum[i][k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    typename SideA::F af[2][FB];
    typename SideB::F bf[2][FA];
    // fragment f of half h of block b, A's first
    auto read = [&](int f, uint32_t b, int h) {
      const LocalPointer here = (LocalPointer)lds + b % kStages * kStage;
      if (f < FB) af[h][f] = SideA::read(here, SideA::near(at_a, f), h);
      else bf[h][f - FB] = SideB::read(here + SideA::kBytes, SideB::near(at_b, f - FB), h);
    };
    constexpr int kReads = FA + FB, kEarly = FA > 2 ? FA - 2 : 1;
#pragma unroll
    for (int s = 0; s < kStages; ++s) {
      next();
#pragma unroll
      for (int l = 0; l < kLoads; ++l) fetch(l, s);
      left -= kDepth;
    }
    wait_for<(kStages - 1) * kLoads>();
    barrier();
#pragma unroll
    for (int f = 0; f < kReads; ++f) read(f, 0, 0);
#pragma unroll 1
    for (uint32_t b = 0; b < blocks; ++b) {
      also(af[0]);
#pragma unroll
      for (int i = 0; i < FA; ++i) {
#pragma unroll
        for (int f = i * kReads / kEarly; f < (i + 1) * kReads / kEarly && f < kReads; ++f)
          read(f, b, 1);
#pragma unroll
        for (int k = 0; k < FB; ++k) sum[i][k] = multiply(bf[0][i], af[0][k], sum[i][k]);
        __builtin_amdgcn_sched_barrier(0);
      }
      wait_for<(kStages - 2) * kLoads>();
      barrier();  // block b has been read, and block b + 1 is there
      next();
      also(af[1]);
#pragma unroll
      for (int i = 0; i < FA; ++i) {
#pragma unroll
        for (int l = i * kLoads / FA; l < (i + 1) * kLoads / FA; ++l)
          fetch(l, b % kStages);
#pragma unroll
        for (int f = i * kReads / kEarly; f < (i + 1) * kReads / kEarly && f < kReads; ++f)
          read(f, b + 1, 0);
#pragma unroll
        for (int k = 0; k < FB; ++k) sum[i][k] = multiply(bf[1][i], af[1][k], sum[i][k]);
        __builtin_amdgcn_sched_barrier(0);
      }
      left -= kDepth;
    }
    wait_for<0>();
    barrier();  // LDS is free
  }

  // Every output of the first `lines` x `columns`, N neighbouring ones of a line at a time, 16
  // bytes of the result: ask(state, line, column), and some lines later put(state, line, column,
  // values); the line's last ones, fewer than N, some(line, column, how many, value by number). A
  // lane has four columns of one line in each of its sums; by way of the wave's own part of LDS,
  // `kPass` sums at a time, they become lines of FA * 16 columns, in 16-byte pieces: for N = 8 the
  // even ones, then the odd ones. Piece p lies at p ^ line % kSwap. So 16 lanes that write a piece
  // of 16 lines, or read 16 pieces (every other one) of a line, have banks of their own.
  // (Eight fp32 values a lane, in two stores of 16 bytes each: 19 workers' 16384 x 2048 x 8192 took
  // 710 us, four with every store whole lines 668.)
  template <int N, typename State, typename Ask, typename Put, typename Some>
  static __device__ __forceinline__ void rows_of(uint8_t* lds, const v4f (&sum)[FA][FB],
                                                 int64_t lines, int64_t columns, Ask&& ask,
                                                 Put&& put, Some&& some) {
    constexpr int kLine = FA * 64, kRoom = 2 * kStage / kWaves;
    constexpr int kPass = kRoom / (16 * kLine) < FB ? kRoom / (16 * kLine) : FB;
    constexpr int kInLine = FA * 16 / N, kSwap = FA * 4 < 16 ? FA * 4 : 16, kApart = 64 / kInLine;
    constexpr int kSteps = kPass * 16 / kApart;  // of a pass
    constexpr int kAsked = kSteps % 2 == 0 ? 2 : 1;
    static_assert(kPass > 0 && FB % kPass == 0 && (N == 4 || N == 8), "equal parts");
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int wj = wave / WM, wm = wave % WM;
    uint8_t* const own = lds + wave * kRoom;
    const int first = lane / kInLine, c = lane % kInLine, column = wj * FA * 16 + c * N;
    const int here = lines < kRows ? static_cast<int>(lines) : kRows;
    const int left = columns - column < N ? static_cast<int>(columns - column) : N;
    // where piece p of a line lies
    auto place = [](int p, int line) {
      const int at = N == 8 ? p / 2 + FA * 2 * (p % 2) : p;
      return line * kLine + (at ^ (line % kSwap)) * 16;
    };
    State state[kAsked];
#pragma unroll
    for (int q = 0; q < kAsked; ++q) {
      const int line = wm * FB * 16 + first + q * kApart;
      if (left == N && line < here) ask(state[q], line, column);
    }
#pragma unroll
    for (int k0 = 0; k0 < FB; k0 += kPass) {
#pragma unroll
      for (int k = 0; k < kPass; ++k)
#pragma unroll
        for (int i = 0; i < FA; ++i)
          *reinterpret_cast<v4f*>(own + place(i * 4 + lane / 16, k * 16 + lane % 16)) =
              sum[i][k0 + k];
      wave_exchange();
#pragma unroll 1
      for (int r0 = first; r0 < kPass * 16; r0 += kAsked * kApart) {
#pragma unroll
        for (int q = 0; q < kAsked; ++q) {
          const int r = r0 + q * kApart, line = (wm * FB + k0) * 16 + r;
          if (line >= here || left <= 0) continue;
          auto piece = [&](int e) {
            return reinterpret_cast<const float*>(own + place(c * (N / 4) + e, r));
          };
          if (left < N) {
            some(line, column, left, [&](int e) { return piece(e / 4)[e % 4]; });
            continue;
          }
          float t[N];
#pragma unroll
          for (int e = 0; e < N / 4; ++e) {
            const v4f v = *reinterpret_cast<const v4f*>(piece(e));
#pragma unroll
            for (int f = 0; f < 4; ++f) t[e * 4 + f] = v[f];
          }
          const State now = state[q];
          const int later = line + kAsked * kApart;
          if (later < here && later < (wm + 1) * FB * 16) ask(state[q], later, column);
          put(now, line, column, t);
        }
      }
      wave_exchange();
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

struct Nothing {};

template <bool PAST_CACHES = false>
__device__ __forceinline__ void store_four(float* to, const float* v) {
  typedef float Four __attribute__((ext_vector_type(4), aligned(4)));
  const Four t = {v[0], v[1], v[2], v[3]};
  if constexpr (PAST_CACHES) __builtin_nontemporal_store(t, reinterpret_cast<Four*>(to));
  else *reinterpret_cast<Four*>(to) = t;
}

template <typename T, bool AA, bool BA, int WJ, int WM, int FA, int FB>
__global__ __launch_bounds__(64 * WJ * WM) void k_product(Job p, Epilogue to) {
  typedef Tile<T, AA, BA, WJ, WM, FA, FB> Of;
  __shared__ __align__(1024) uint8_t lds[Of::kLds];
  const Place at = place_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_j);
  const int64_t m0 = at.m * Of::kRows, j0 = at.j * Of::kCols, k0 = at.part * p.share;
  const Parts<T> parts = {static_cast<const T*>(p.a) + (AA ? k0 * p.lda + m0 : m0 * p.lda + k0),
                          static_cast<const T*>(p.b) + (BA ? k0 * p.ldb + j0 : j0 * p.ldb + k0),
                          p.rows - m0, p.cols - j0,
                          p.depth - k0 < p.share ? p.depth - k0 : p.share};
  v4f sum[FA][FB];
  Of::sums(lds, p.lda, p.ldb, parts, sum, [](auto&) {});
  if (p.partial) {  // whose lines go on to whole eights
    float* const out = p.partial + at.part * p.rows * p.ld_partial + m0 * p.ld_partial + j0;
    Of::template rows_of<4, Nothing>(
        lds, sum, parts.rows, (parts.cols + 7) / 8 * 8, [](Nothing&, int, int) {},
        [&](const Nothing&, int line, int column, float* v) {
          store_four(out + line * p.ld_partial + column, v);
        },
        [](int, int, int, auto&&) {});
  } else {
    constexpr int kPiece = 16 / sizeof(T);
    typedef Finish<T, kPiece> Piece;
    Of::template rows_of<kPiece, Piece>(
        lds, sum, parts.rows, parts.cols,
        [&](Piece& f, int line, int column) { f.ask(to, m0 + line, j0 + column); },
        [&](const Piece& f, int line, int column, float* v) {
          f.put(to, m0 + line, j0 + column, v);
        },
        [&](int line, int column, int left, auto&& value) {
          Piece::some(to, m0 + line, j0 + column, left, value);
        });
  }
}

// Few rows (up to 16), B along: the time is B's bytes, or latency where they are few (one
// token, 4096 x 4096 in bf16: 8 us, 4.2 TB/s, against 8.7 + 4.8 us in tiles with shares). A
// workgroup takes 16 columns, its waves every WAVES-th block each, fragments straight from memory
// and several blocks at a time; the waves' sums meet in LDS, added in one order. Any address and
// distance of rows is taken.
template <typename T, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_product_few(Job p, Epilogue to) {
  typedef typename Fragment<T>::type F;
  typedef T Loose __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
  constexpr int kAtOnce = 4, kDepth = 128 / sizeof(T), kPiece = 16 / sizeof(T);
  __shared__ v4f sums[WAVES][64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int64_t j0 = static_cast<int64_t>(blockIdx.x) * 16;
  const int64_t line = j0 + lane % 16 < p.cols ? j0 + lane % 16 : p.cols - 1;
  const T* const from_b = static_cast<const T*>(p.b) + line * p.ldb;
  const int64_t m = lane % 16 < p.rows ? lane % 16 : p.rows - 1;
  const T* const from_a = static_cast<const T*>(p.a) + m * p.lda;
  v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
  const int64_t c0 = lane / 16 * kPiece;
  auto whole_piece = [&](const T* q, int64_t c) {
    const Loose t = *reinterpret_cast<const Loose*>(q + c);
    F v;
#pragma unroll
    for (int e = 0; e < kPiece; ++e) v[e] = t[e];
    return v;
  };
  auto some_piece = [&](const T* q, int64_t c) {  // zeros past the depth
    F v;
#pragma unroll
    for (int e = 0; e < kPiece; ++e) v[e] = c + e < p.depth ? q[c + e] : static_cast<T>(0.0f);
    return v;
  };
  const int blocks = static_cast<int>((p.depth + kDepth - 1) / kDepth);
  const int whole_blocks = static_cast<int>(p.depth / kDepth);
  int b0 = wave;
  for (; b0 + (kAtOnce - 1) * WAVES < whole_blocks; b0 += WAVES * kAtOnce) {
    F bf[kAtOnce][2], af[kAtOnce][2];
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t c = (b0 + u * WAVES) * int64_t{kDepth} + h * 4 * kPiece + c0;
        bf[u][h] = whole_piece(from_b, c);
        af[u][h] = whole_piece(from_a, c);
      }
    }
#pragma unroll
    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) sum = multiply(bf[u][h], af[u][h], sum);
  }
  for (; b0 < blocks; b0 += WAVES) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int64_t c = b0 * int64_t{kDepth} + h * 4 * kPiece + c0;
      const bool there = b0 < whole_blocks;
      sum = multiply(there ? whole_piece(from_b, c) : some_piece(from_b, c),
                     there ? whole_piece(from_a, c) : some_piece(from_a, c), sum);
    }
  }
  sums[wave][lane] = sum;
  __syncthreads();
  const int64_t j = j0 + lane / 16 * 4;
  if (wave > 0 || lane % 16 >= p.rows) return;
  v4f all = sums[0][lane];
#pragma unroll
  for (int i = 1; i < WAVES; ++i) all += sums[i][lane];
  float v[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = all[e];
  if (j + 4 <= p.cols) {
    Finish<T, 4> f;
    f.ask(to, m, j);
    f.put(to, m, j, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e >= p.cols) break;
      Finish<T, 1> f;
      f.ask(to, m, j + e);
      f.put(to, m, j + e, v + e);
    }
  }
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
  if (j + 8 <= p.cols) {
    Finish<T, 8> f;
    f.ask(to, m, j);
    f.put(to, m, j, sum);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (j + e >= p.cols) break;
      Finish<T, 1> f;
      f.ask(to, m, j + e);
      f.put(to, m, j + e, sum + e);
    }
  }
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
                                                                 int64_t ld_dbias,
                                                                 bool whole_lines) {
  typedef Tile<T, true, true, WJ, WM, FA, FB> Of;
  __shared__ __align__(1024) uint8_t lds[Of::kLds];
  const Place at = place_of(blockIdx.x, gridDim.x, p.tiles_m, p.tiles_j);
  const int64_t m0 = at.m * Of::kRows, j0 = at.j * Of::kCols;
  const int worker = at.part % w.n;
  int64_t t0 = w.first[worker], end = w.first[worker + 1];
  const int64_t blocks = (end - t0 + Of::kDepth - 1) / Of::kDepth;
  const int64_t most = (blocks + w.splits - 1) / w.splits * Of::kDepth;
  t0 += at.part / w.n * most;
  end = t0 + most < end ? t0 + most : end;
  const Parts<T> parts = {static_cast<const T*>(p.a) + t0 * p.lda + m0,
                          static_cast<const T*>(p.b) + t0 * p.ldb + j0, p.rows - m0, p.cols - j0,
                          end > t0 ? end - t0 : 0};
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int wj = wave / WM, wm = wave % WM;
  typename Fragment<T>::type one;
#pragma unroll
  for (int e = 0; e < static_cast<int>(16 / sizeof(T)); ++e) one[e] = static_cast<T>(1.0f);
  v4f sum[FA][FB], ones[FB];
#pragma unroll
  for (int k = 0; k < FB; ++k) ones[k] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  // the sums of dy's columns are made by the tiles of the first inputs
  const bool with_bias = dbias && j0 == 0 && wj == 0;
  Of::sums(lds, p.lda, p.ldb, parts, sum, [&](auto& af) {
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
  // Whole lines go past the caches: with 19 workers' 16384 x 4096 x 4096 674 us by way of them and
  // 596 past them, with 11 workers' 1000 x 4096 x 4096 176 and 148 (1000 x 2048 x 2048, which the
  // caches hold, 48 and 51). (Lines of several tiles of one row next to each other matter too: four
  // tiles deep 16384 x 2048 x 8192 takes 667, eight 700.)
  float* const out = dw + at.part * ld_dw + m0 * p.cols + j0;
  auto store = [&](auto past_caches) {
    Of::template rows_of<4, Nothing>(
        lds, sum, parts.rows, parts.cols, [](Nothing&, int, int) {},
        [&](const Nothing&, int line, int column, float* v) {
          store_four<decltype(past_caches)::value>(out + line * p.cols + column, v);
        },
        [&](int line, int column, int left, auto&& value) {
#pragma unroll 1
          for (int e = 0; e < left; ++e) out[line * p.cols + column + e] = value(e);
        });
  };
  if (whole_lines) store(std::true_type());
  else store(std::false_type());
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

// Matrices once more, with rows of whole 16-byte pieces (the last one's rest 0): the first
// `groups` workgroups the first one, the others the second.
struct Packed {
  const void* from;
  int64_t ld, rows, cols;
  void* to;
  int64_t ld_to;
};
template <typename T>
__global__ __launch_bounds__(kBlock) void k_pack_rows(Packed first, Packed second, uint32_t groups) {
  constexpr int kPiece = 16 / sizeof(T);
  typedef T Piece __attribute__((ext_vector_type(kPiece)));
  typedef T Loose __attribute__((ext_vector_type(kPiece), aligned(sizeof(T))));
  const bool later = blockIdx.x >= groups;
  const Packed m = later ? second : first;
  const int64_t pieces = m.ld_to / kPiece, group = later ? blockIdx.x - groups : blockIdx.x;
  const int64_t all = later ? gridDim.x - groups : groups;
  for (int64_t i = group * kBlock + threadIdx.x; i < m.rows * pieces; i += all * kBlock) {
    const int64_t r = i / pieces, c = i % pieces * kPiece;
    const T* p = static_cast<const T*>(m.from) + r * m.ld + c;
    Piece v;
    if (c + kPiece <= m.cols) {
      v = *reinterpret_cast<const Loose*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < kPiece; ++e) v[e] = c + e < m.cols ? p[e] : static_cast<T>(0.0f);
    }
    *reinterpret_cast<Piece*>(static_cast<T*>(m.to) + i * kPiece) = v;
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

constexpr int64_t kMaxApart = int64_t{1} << 22;  // bytes between rows: 256 are within 2^30

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

// The matrix as the product reads it: as it is, or its place in the workspace (`rest`: from here
// on), to be packed there.
template <typename T>
Packed whole(const void* p, int64_t* ld, int64_t rows, int64_t cols, char** rest) {
  Packed m = {p, *ld, rows, cols, nullptr, 0};
  if (is_whole(p, *ld, rows, cols, sizeof(T))) {
    if (rows < 2) *ld = cols;
  } else {
    m.to = *rest;
    *ld = m.ld_to = up_to(cols, 16 / sizeof(T));
    *rest += packed_bytes(rows, cols, sizeof(T));
  }
  return m;
}

// Packs what has to be, and gives where both are then.
template <typename T>
void pack(const Packed& a, const Packed& b, const void** at_a, const void** at_b, hipStream_t s) {
  auto groups = [](const Packed& m) {
    const int64_t g = m.to ? (m.rows * (m.ld_to * sizeof(T) / 16) + kBlock - 1) / kBlock : 0;
    return static_cast<uint32_t>(std::min(g, int64_t{1} << 22));
  };
  const uint32_t first = groups(a), second = groups(b);
  if (first + second > 0)
    launch("pack_rows", k_pack_rows<T>, dim3(first + second), dim3(kBlock), 0, s, a, b, first);
  *at_a = a.to ? a.to : a.from;
  *at_b = b.to ? b.to : b.from;
}

int64_t tiles_of(int64_t rows, int64_t cols, int size) {
  return ((rows + size - 1) / size) * ((cols + size - 1) / size);
}

// Tiles of 64, 128 or 256 lines (32: of 32 rows x 64 columns), and into how many shares their
// depth is cut.
struct Plan {
  int size, shares;
  int64_t share;  // depths
};

// The tiles, of n matrices, with the least work for the busiest CU, an output of small tiles weighed
// as more. An fp32 tile takes its products' time, whatever its neighbours (6724 x 2560 x 1808, 270
// tiles of 256 or 4240 of 64: 851 us and 477; 777 x 1500 x 1000, 312 of 64 or 600 of 32: 41 and 34). One
// of 16 bits is bound by what it reads, too: 7476 x 1104 x 3984 in bf16, 150 tiles of 256 or 531 of
// 128, 94 us and 130; 2048 x 4096 x 4096, 128 of 256 or 512 of 128, 84 and 64; 1000 x 2000 x 3000, 128 of
// 128 or 512 of 64, 43 and 30; 18 workers' 879 x 3600 x 128, 270 of 256 or 522 of 128, 17 and 13 (2052
// of 64 would take 11).
int least_work(int64_t rows, int64_t cols, int64_t n, int64_t size, bool halves) {
  const int64_t cus = device_cus();
  int64_t least = INT64_MAX;
  int best = 64;
  auto weigh = [&](int tile, int64_t tiles, int64_t outputs, int64_t percent) {
    const int64_t work = (tiles * n + cus - 1) / cus * outputs * percent;
    if (work < least) {
      least = work;
      best = tile;
    }
  };
  const bool f32 = size == 4;
  if (halves) weigh(32, (rows + 31) / 32 * ((cols + 63) / 64), 32 * 64, 112);
  weigh(64, tiles_of(rows, cols, 64), 64 * 64, f32 ? 105 : 200);
  weigh(128, tiles_of(rows, cols, 128), 128 * 128, 100);
  weigh(256, tiles_of(rows, cols, 256), 256 * 256, f32 ? 95 : 65);
  return best;
}

// Few tiles of much depth are cut into equal shares of ten blocks or more, the last one of what is left,
// up to two for a CU: in bf16 128 x 512 x 8192 takes 13.3 us in twelve, 37.8 whole, 300 x 1000 x 4096
// 14.8 in six, 21.1 whole.
Plan plan_product(int64_t rows, int64_t cols, int64_t depth, int64_t size) {
  const int64_t block = 128 / size, blocks = (depth + block - 1) / block;
  Plan p = {64, 1, (blocks > 0 ? blocks : 1) * block};
  const int64_t cus = device_cus(), tiles = tiles_of(rows, cols, 64);
  const int64_t want = tiles > 0 ? std::min(2 * cus / tiles, blocks / 10) : 1;
  if (want >= 2) {
    const int64_t per = (blocks + want - 1) / want;
    p.share = per * block;
    p.shares = static_cast<int>((blocks + per - 1) / per);
  } else {
    p.size = least_work(rows, cols, 1, size, size == 4);
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

// Whether the matrix's rows are whole lines, which are stored past the caches: 16384 x 8192 x 2048
// with gelu and p takes 557 us so and 559 to 575 by way of them. Parts of lines stay for the others.
bool whole_lines(const void* p, int64_t ld, int64_t size) {
  return reinterpret_cast<uintptr_t>(p) % 128 == 0 && ld * size % 128 == 0;
}

template <typename T, bool BA>
void choose_product(const Product& of, void* workspace, hipStream_t s) {
  char* rest = static_cast<char*>(workspace);
  Job p = {};
  p.lda = of.a.ld;
  p.ldb = of.b.ld;
  const Packed a = whole<T>(of.a.p, &p.lda, of.rows, of.depth, &rest);
  const Packed b = BA ? whole<T>(of.b.p, &p.ldb, of.depth, of.cols, &rest)
                      : whole<T>(of.b.p, &p.ldb, of.cols, of.depth, &rest);
  pack<T>(a, b, &p.a, &p.b, s);
  p.rows = of.rows;
  p.cols = of.cols;
  p.depth = of.depth;
  const Plan plan = plan_product(p.rows, p.cols, p.depth, sizeof(T));
  Epilogue to = of.to;
  to.past_caches = whole_lines(to.out, to.ld_out, sizeof(T)) &&
                   (!to.pre || whole_lines(to.pre, to.ld_pre, sizeof(T)));
  p.share = plan.share;
  if (plan.shares > 1) {
    to.past_caches = false;  // k_finish
    p.partial = reinterpret_cast<float*>(rest);
    p.ld_partial = up_to(p.cols, 8);
  }
  if (plan.size == 256) launch_tiles<T, BA, 2, 4, 8, 4>(p, plan, to, s);
  else if (plan.size == 128) launch_tiles<T, BA, 2, 2, 4, 4>(p, plan, to, s);
  else if (plan.size == 64) launch_tiles<T, BA, 2, 2, 2, 2>(p, plan, to, s);
  else if constexpr (sizeof(T) == 4) launch_tiles<T, BA, 2, 2, 2, 1>(p, plan, to, s);
  if (plan.shares > 1)
    launch("finish", k_finish<T>,
           dim3(static_cast<uint32_t>((p.rows * (p.ld_partial / 8) + kBlock - 1) / kBlock)),
           dim3(kBlock), 0, s, p, plan.shares, to);
}

// Up to this many rows, and B along, the form for few: 16 x 4096 x 4096 in bf16 takes 9.7 us so
// and 12.4 in tiles with shares, 32 rows in two such fragments 13.4 and in tiles 13.0.
constexpr int64_t kFew = 16;
bool is_few(const Product& p) { return !p.b.across && p.rows <= kFew; }

template <typename T, int WAVES>
void launch_few(const Product& of, hipStream_t s) {
  Job p = {};
  p.a = of.a.p;
  p.b = of.b.p;
  p.lda = of.a.ld;
  p.ldb = of.b.ld;
  p.rows = of.rows;
  p.cols = of.cols;
  p.depth = of.depth;
  launch("product_few", k_product_few<T, WAVES>,
         dim3(static_cast<uint32_t>((p.cols + 15) / 16)), dim3(64 * WAVES), 0, s, p, of.to);
}

// As many waves as there are blocks for, up to 16.
template <typename T>
void choose_few(const Product& p, hipStream_t s) {
  constexpr int64_t kDepth = 128 / sizeof(T);
  if (p.depth > 16 * kDepth) launch_few<T, 16>(p, s);
  else if (p.depth > 4 * kDepth) launch_few<T, 8>(p, s);
  else launch_few<T, 4>(p, s);
}

template <typename T>
void launch_product(const Product& p, void* workspace, hipStream_t s) {
  if (is_few(p)) {
    choose_few<T>(p, s);
    return;
  }
  if (p.b.across) choose_product<T, true>(p, workspace, s);
  else choose_product<T, false>(p, workspace, s);
}

// As plan_product, of every worker's gradient: the depth is its tokens.
Plan plan_gradient(const DenseGradient& a, int64_t size) {
  const int64_t block = 128 / size, blocks = (a.tokens / a.n + block - 1) / block;
  Plan p = {64, 1, 0};
  const int64_t tiles = tiles_of(a.outputs, a.inputs, 64) * a.n;
  const int64_t want = tiles > 0 ? std::min(3 * int64_t{device_cus()} / tiles, blocks / 4) : 1;
  if (want >= 2) p.shares = static_cast<int>(std::min<int64_t>(want, 16));
  else p.size = least_work(a.outputs, a.inputs, a.n, size, false);
  return p;
}

template <typename T, int WJ, int WM, int FA, int FB>
void launch_gradients(Job p, const Workers& w, float* dw, int64_t ld_dw, float* dbias,
                      int64_t ld_dbias, hipStream_t s) {
  p.tiles_m = static_cast<uint32_t>((p.rows + WM * FB * 16 - 1) / (WM * FB * 16));
  p.tiles_j = static_cast<uint32_t>((p.cols + WJ * FA * 16 - 1) / (WJ * FA * 16));
  const bool whole_lines =
      reinterpret_cast<uintptr_t>(dw) % 128 == 0 && ld_dw % 32 == 0 && p.cols % 32 == 0;
  // A launch has fewer than 2^32 threads: many workers' tiles may take several
  const int64_t tiles = int64_t{p.tiles_m} * p.tiles_j * w.splits;
  const int fit = static_cast<int>(std::min<int64_t>(0xffffffff / (64 * WJ * WM) / tiles, w.n));
  for (int i = 0; i < w.n; i += fit) {
    Workers some = w;
    some.n = w.n - i < fit ? w.n - i : fit;
    for (int k = 0; k <= some.n; ++k) some.first[k] = w.first[i + k];
    launch("dense_gradient", k_dense_gradient<T, WJ, WM, FA, FB>,
           dim3(static_cast<uint32_t>(tiles * some.n)), dim3(64 * WJ * WM), 0, s, p, some,
           dw + i * ld_dw, ld_dw, dbias ? dbias + i * ld_dbias : nullptr, ld_dbias, whole_lines);
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
  const Packed dy = whole<T>(a.dy, &p.lda, a.tokens, a.outputs, &rest);
  const Packed x = whole<T>(a.x, &p.ldb, a.tokens, a.inputs, &rest);
  pack<T>(dy, x, &p.a, &p.b, s);
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
  if (is_few(p)) return 0;
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
