// Dense layers on rows: y = alpha act(x W' + b) + residual, and the gated block's h = act(x Wg' + bg) (x Wu' + bu), with their gradients.
//
// Backward, with z the products plus their biases: dz = alpha dy act'(z) (gated: dg = dh u act'(g), du = dh act(g)), then dx = dz W,
// dW = dz' x, db = sum over the rows of dz.  dz is an operand of the matrix units and so rounded to the operands' type (of few values: the sum of
// two numbers of it); db is summed from it before that.  z is either what the forward call kept, in 32 bits, or computed again.
//
// All products are tiles of C = A B' (products.h): A has the columns of the result, so that a lane's registers hold neighbouring ones, and B
// its rows.  The gated product's two weights are one operand with 32 rows of each in turn: a wave has the gate's and the up projection's sums
// of the same elements, and x is read once for both.  A tile leaves its sums through LDS, so that what follows reads and writes whole rows.
// Where there are few tiles for the chip, k is split: the parts are left in 32 bits and a second kernel adds them up, in their order, ahead
// of the same epilogue.
#include <atomic>
#include <type_traits>
#include <utility>

#include "activations.h"
#include "coop_internal.h"
#include "dealing.h"
#include "products.h"

namespace coop {
namespace {

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }
int64_t at_most(int64_t x, int64_t most) { return x < 1 ? 1 : x < most ? x : most; }

// f of 0 .. N - 1 as compile-time constants: a loop that indexes registers, whatever is in it
template <typename F, int... I>
__device__ __forceinline__ void each_of(F&& f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each_of(F&& f) {
  each_of(f, std::make_integer_sequence<int, N>());
}

template <int T> constexpr int kE = 16 / kElem<T>;  // elements of a pack of 16 bytes

// Columns col .. col + E - 1 of a row of `dim`: those that there are; the others read as zeros.
template <int T, int E>
__device__ __forceinline__ void load_columns(const void* row, int32_t col, int32_t dim, float (&f)[E]) {
  typedef typename Element<T>::M M;
  const M* p = (const M*)row + col;
  if (col + E <= dim) {
    load_elements<T, E>(p, f);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = col + e < dim ? (float)p[e] : 0.f;
  }
}
template <int T, int E>
__device__ __forceinline__ void store_columns(void* row, int32_t col, int32_t dim, const float (&f)[E]) {
  typedef typename Element<T>::M M;
  M* p = (M*)row + col;
  if (col + E <= dim) {
    store_elements<T, E>(p, f);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (col + e < dim) p[e] = (M)f[e];
  }
}

// what a value loses when it is rounded to the type
template <int T>
__device__ __forceinline__ float lost_to(float v) {
  const float r = v - (float)(typename Element<T>::M)v;
  return fabsf(r) < __builtin_inff() ? r : 0.f;  // (what is not finite, or not in the type, has none)
}

// ---- what becomes of a product's sums --------------------------------------------------------------------------------------
// put(lane, row, v, u): E neighbouring columns of a row of the first product, and of a pair's second.  A lane keeps its columns.

// the forward result
template <int T, bool PAIR>
struct Forward {
  static constexpr bool kSums = false;
  const char *bias, *bias2, *residual;
  float *pre, *pre2;  // null: not kept
  char* out;
  int64_t rows;
  int32_t cols;
  float alpha;
  int act;
  template <int E>
  struct Lane {
    int32_t col;
    float b[E], b2[E];
  };
  template <int E>
  __device__ __forceinline__ void begin(Lane<E>& l, int32_t col) const {
    l.col = col;
#pragma unroll
    for (int e = 0; e < E; ++e) l.b[e] = l.b2[e] = 0.f;
    if (bias != nullptr) load_columns<T, E>(bias, col, cols, l.b);
    if (PAIR && bias2 != nullptr) load_columns<T, E>(bias2, col, cols, l.b2);
  }
  template <int E>
  __device__ __forceinline__ void put(Lane<E>& l, int64_t row, float (&v)[E], float (&u)[E]) const {
    if (row >= rows || l.col >= cols) return;
    const int64_t at = row * cols;
    if (bias != nullptr) {
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += l.b[e];
    }
    if (PAIR && bias2 != nullptr) {
#pragma unroll
      for (int e = 0; e < E; ++e) u[e] += l.b2[e];
    }
    if (pre != nullptr) {
      store_columns<COOP_F32, E>(pre + at, l.col, cols, v);
      if (PAIR) store_columns<COOP_F32, E>(pre2 + at, l.col, cols, u);
    }
    if (out == nullptr) return;  // (computed again, for its gradient)
    act_values(v, act);
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= PAIR ? u[e] : alpha;
    if (!PAIR && residual != nullptr) {
      float r[E];
      load_columns<T, E>(residual + at * kElem<T>, l.col, cols, r);
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += r[e];
    }
    store_columns<T, E>(out + at * kElem<T>, l.col, cols, v);
  }
};

// dz of what the forward product is once more, as an operand (rows of `ld` elements, zeros up to the next pack behind `cols`; a pair's
// second part begins at `second`), and the sums of its columns over the rows that a wave has.
template <int T, bool PAIR>
struct Slope {
  static constexpr bool kSums = true;
  const char *bias, *bias2, *dout;
  char* dz;
  float *part, *part2;  // [waves of rows][cols], or null
  int64_t rows, ld, second;
  int32_t cols;
  float alpha, into;  // (the factor, and what of it is multiplied into dz)
  int act;
  int64_t rest;  // bytes from dz to what it lost to its type, in the same row; 0: that is not kept
  template <int E>
  struct Lane {
    int32_t col;
    float b[E], b2[E], s[E], s2[E];
  };
  template <int E>
  __device__ __forceinline__ void begin(Lane<E>& l, int32_t col) const {
    l.col = col;
#pragma unroll
    for (int e = 0; e < E; ++e) l.b[e] = l.b2[e] = l.s[e] = l.s2[e] = 0.f;
    if (bias != nullptr) load_columns<T, E>(bias, col, cols, l.b);
    if (PAIR && bias2 != nullptr) load_columns<T, E>(bias2, col, cols, l.b2);
  }
  // v, u: the products' sums with their biases (behind the last column: anything); they are lost
  template <int E>
  __device__ __forceinline__ void slope(Lane<E>& l, int64_t row, float (&v)[E], const float (&u)[E]) const {
    float d[E], d2[E], value[E];
    load_columns<T, E>(dout + row * cols * kElem<T>, l.col, cols, d);
    act_slopes(v, value, act);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const bool there = l.col + e < cols;
      if (PAIR) {
        d2[e] = there ? d[e] * value[e] : 0.f;
        d[e] = there ? d[e] * u[e] * v[e] : 0.f;
        l.s2[e] += d2[e];
        l.s[e] += d[e];
      } else {  // (without an activation dz is the gradient as it came)
        l.s[e] += there ? d[e] * alpha * v[e] : 0.f;
        if (act != COOP_ACT_NONE) d[e] = there ? d[e] * into * v[e] : 0.f;
      }
    }
    if (dz == nullptr) return;
    store_elements<T, E>(dz + (row * ld + l.col) * kElem<T>, d);
    if (PAIR) store_elements<T, E>(dz + (row * ld + second + l.col) * kElem<T>, d2);
    if (T == COOP_F32 || rest == 0) return;
#pragma unroll
    for (int e = 0; e < E; ++e) d[e] = lost_to<T>(d[e]), d2[e] = PAIR ? lost_to<T>(d2[e]) : 0.f;
    store_elements<T, E>(dz + rest + (row * ld + l.col) * kElem<T>, d);
    if (PAIR) store_elements<T, E>(dz + rest + (row * ld + second + l.col) * kElem<T>, d2);
  }
  template <int E>
  __device__ __forceinline__ void put(Lane<E>& l, int64_t row, float (&v)[E], float (&u)[E]) const {
    if (row >= rows || l.col >= cols) return;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] += l.b[e], u[e] += PAIR ? l.b2[e] : 0.f;
    slope(l, row, v, u);
  }
  // the lanes of a wave whose numbers differ in the bits from `lanes` on have the same columns
  template <int E>
  __device__ __forceinline__ void end(Lane<E>& l, int lanes, int64_t part_row) const {
    if (part == nullptr) return;
#pragma unroll
    for (int e = 0; e < E; ++e)
      for (int off = lanes; off < kWave; off <<= 1) {
        l.s[e] += __shfl_xor(l.s[e], off, kWave);
        if (PAIR) l.s2[e] += __shfl_xor(l.s2[e], off, kWave);
      }
    if (lane_id() >= lanes || l.col >= cols) return;
    store_columns<COOP_F32, E>(part + part_row * cols, l.col, cols, l.s);
    if (PAIR) store_columns<COOP_F32, E>(part2 + part_row * cols, l.col, cols, l.s2);
  }
};

// a gradient, times `scale`; rows from `second` on are another array's (each has `rows` of them)
struct Gradient {
  static constexpr bool kSums = false;
  char *out, *out2;
  int64_t rows, second;
  int32_t cols;
  float scale;
  int type;
  template <int E> struct Lane { int32_t col; };
  template <int E>
  __device__ __forceinline__ void begin(Lane<E>& l, int32_t col) const { l.col = col; }
  template <int E>
  __device__ __forceinline__ void put(Lane<E>& l, int64_t row, float (&v)[E], float (&)[E]) const {
    char* to = out;
    if (out2 != nullptr && row >= second) row -= second, to = out2;
    if (row >= rows || l.col >= cols) return;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] *= scale;
    if (type == COOP_F32) store_columns<COOP_F32, E>(to + row * cols * 4, l.col, cols, v);
    else if (type == COOP_F16) store_columns<COOP_F16, E>(to + row * cols * 2, l.col, cols, v);
    else store_columns<COOP_BF16, E>(to + row * cols * 2, l.col, cols, v);
  }
};

// a split's part: [split][rows][width], of a pair the second product `width / 2` columns behind the first
template <bool PAIR>
struct Part {
  static constexpr bool kSums = false;
  float* sums;
  int64_t rows, width, split_rows;
  template <int E> struct Lane { int32_t col; };
  template <int E>
  __device__ __forceinline__ void begin(Lane<E>& l, int32_t col) const { l.col = col; }
  template <int E>
  __device__ __forceinline__ void put(Lane<E>& l, int64_t row, float (&v)[E], float (&u)[E]) const {
    const int64_t half = PAIR ? width / 2 : width;
    if (row >= rows || l.col >= half) return;
    float* to = sums + (split_rows + row) * width + l.col;
    store_elements<COOP_F32, E>(to, v);
    if (PAIR) store_elements<COOP_F32, E>(to + half, u);
  }
};

// ---- products ------------------------------------------------------------------------------------------------------------------
// FORM: one operand A; a pair of them (their rows in turn); or two, one behind the other along k, where B's k goes on.
enum { kOne, kPair, kTwo };

// Which tiles a block has: those of a split are dealt out in strips of kStrip of B's, so that the 32 blocks that an XCD runs at a time have
// neighbouring ones of both operands.
constexpr uint32_t kStrip = 4;
struct Tiles {
  uint32_t a, b, splits;
  struct Mine { uint32_t a, b, split; };
  __device__ __forceinline__ Mine mine() const {
    const uint32_t i = xcd_runs(blockIdx.x, gridDim.x), split = i / (a * b), t = i - split * (a * b);
    const uint32_t first = t / (a * kStrip) * kStrip, at = t - first * a, rows = b - first < kStrip ? b - first : kStrip;
    return Mine{at / rows, first + at % rows, split};
  }
};

// TWICE: B with what is added to it.
template <int T, int WA, int WB, int TA, int TB, bool SA, bool SB, int SIZE, int FORM, bool TWICE, typename Fin>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_dense(Operand a, Operand a2, Operand b, Operand b2, int64_t k,
                                                                                               Tiles tiles, Fin fin) {
  typedef Product<T, WA, WB, TA, TB, SA, SB, SIZE, FORM == kPair, TWICE> P;
  extern __shared__ char lds[];
  constexpr int kColsA = FORM == kPair ? P::kRowsA / 2 : P::kRowsA;  // of the result
  const Tiles::Mine mine = tiles.mine();
  const int64_t col0 = (int64_t)mine.a * kColsA, row0 = (int64_t)mine.b * P::kRowsB;
  const int64_t stages = (k + P::kK - 1) / P::kK;
  const int64_t k0 = stages * mine.split / tiles.splits * P::kK, k1 = stages * (mine.split + 1) / tiles.splits * P::kK;
  P p;
  if constexpr (FORM == kTwo) {
    p.begin_two(a, b, a2, b2, col0, row0, k0, k1, lds);
    p.zero();
    p.tile();
    p.last();
    p.tile();
  } else {
    p.begin(a, b, col0, row0, k0, k1, 0, lds);
    p.zero();
    p.tile();
  }
  P::end();
  if constexpr (std::is_same<Fin, Part<FORM == kPair>>::value) fin.split_rows = mine.split * fin.rows;
  // Through LDS, a wave for itself: 32 rows at a time, written by columns, read by rows.
  constexpr int E = kE<T>, kLdsCols = TA * 32, kCols = FORM == kPair ? kLdsCols / 2 : kLdsCols, kRow = kLdsCols + 4;  // (rows begin in different banks)
  constexpr int kLanes = kCols / E, kEach = kWave / kLanes;  // lanes of a row, rows at a time
  static_assert(P::kWaves * 32 * kRow * 4 <= P::kLds && kLanes <= kWave, "the waves' rows lie where the stages were");
  float* const own = reinterpret_cast<float*>(lds) + uniform_wave_in_block() * (32 * kRow);
  const int lane = lane_id(), mine_col = lane % kLanes * E;
  typename Fin::template Lane<E> at;
  fin.begin(at, (int32_t)(col0 + P::a0() / (kLdsCols / kCols)) + mine_col);
  each_of<TB>([&](auto number) {
    constexpr int j = decltype(number)::value;
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f[4] = {p.acc[i][j][4 * q], p.acc[i][j][4 * q + 1], p.acc[i][j][4 * q + 2], p.acc[i][j][4 * q + 3]};
        const int col = (FORM == kPair ? (i & 1) * kCols + (i >> 1) * 32 : i * 32) + P::row_of(4 * q) + P::own_row();
        store_elements<COOP_F32, 4>(own + (lane & 31) * kRow + col, f);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 4
    for (int i = 0; i < 32 / kEach; ++i) {
      const int r = i * kEach + lane / kLanes;
      float v[E], u[E];
      load_elements<COOP_F32, E>(own + r * kRow + mine_col, v);
      if constexpr (FORM == kPair) load_elements<COOP_F32, E>(own + r * kRow + kCols + mine_col, u);
      else {
#pragma unroll
        for (int e = 0; e < E; ++e) u[e] = 0.f;
      }
      fin.put(at, row0 + P::b0() + j * 32 + r, v, u);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  });
  if constexpr (Fin::kSums) fin.end(at, kLanes, (int64_t)mine.b * WB + uniform_wave_in_block() % WB);
}

// The splits' parts added up, and the epilogue.  A wave has 64 packs of four columns; where there are many splits the block's waves deal those of
// the same packs among themselves (`share` of them), and the first adds up what they have, in their order.  (512 splits of 128 x 128 by one wave
// each: 41 us.)
constexpr int kSumWaves = 16;
template <int T, bool PAIR, typename Fin>
__global__ __launch_bounds__(kSumWaves* kWave) void k_dense_join(const float* __restrict__ sums, int splits, int share, int64_t rows, int64_t width, int32_t cols,
                                                                 Fin fin) {
  constexpr int E = 4, kValues = PAIR ? 2 * E : E;
  __shared__ float lds[kValues][kSumWaves][kWave];
  const int32_t packs = (cols + E - 1) / E;
  const int64_t half = PAIR ? width / 2 : 0;
  const int wave = uniform_wave_in_block(), lane = lane_id(), mine = wave % share, each = kSumWaves / share * kWave;
  for (int64_t first = (int64_t)blockIdx.x * each; first < rows * packs; first += (int64_t)gridDim.x * each) {
    const int64_t i = first + wave / share * kWave + lane, row = i / packs;
    const int32_t c = (int32_t)(i - row * packs) * E;
    const bool live = row < rows;
    float v[E] = {0.f, 0.f, 0.f, 0.f}, u[E] = {0.f, 0.f, 0.f, 0.f};
    if (live) {
      const float* from = sums + (mine * rows + row) * width + c;
#pragma unroll 8
      for (int q = mine; q < splits; q += share, from += share * rows * width) {
        float f[E];
        load_elements<COOP_F32, E>(from, f);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] += f[e];
        if constexpr (PAIR) {
          load_elements<COOP_F32, E>(from + half, f);
#pragma unroll
          for (int e = 0; e < E; ++e) u[e] += f[e];
        }
      }
    }
    if (share > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < E; ++e) {
        lds[e][wave][lane] = v[e];
        if constexpr (PAIR) lds[E + e][wave][lane] = u[e];
      }
      __syncthreads();
    }
    if (mine != 0 || !live) continue;
    for (int w = 1; w < share; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        v[e] += lds[e][wave + w][lane];
        if constexpr (PAIR) u[e] += lds[E + e][wave + w][lane];
      }
    typename Fin::template Lane<E> at;
    fin.begin(at, c);
    fin.put(at, row, v, u);
  }
}

// dz from what the forward call kept (pre null: there is no activation), or only the sums of its columns (dz null).  2^lanes_log2 lanes share
// a row, blockIdx.x for parts of the columns, blockIdx.y deals the rows; part[blockIdx.y * 4 + wave].
template <int T, bool PAIR>
__global__ __launch_bounds__(kBlock) void k_dense_slope(const float* __restrict__ pre, const float* __restrict__ pre2, int lanes_log2, Slope<T, PAIR> fin) {
  constexpr int E = kE<T>;
  const int lanes = 1 << lanes_log2, lane = lane_id() & (lanes - 1);
  typename Slope<T, PAIR>::template Lane<E> at;
  fin.begin(at, ((int32_t)blockIdx.x * lanes + lane) * E);
  const int64_t step = (int64_t)gridDim.y * (kBlock >> lanes_log2);
  if (at.col < fin.cols) {
#pragma unroll 2
    for (int64_t r = (int64_t)blockIdx.y * (kBlock >> lanes_log2) + (threadIdx.x >> lanes_log2); r < fin.rows; r += step) {
      float v[E], u[E];
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] = u[e] = 0.f;
      if (pre != nullptr) load_columns<COOP_F32, E>(pre + r * fin.cols, at.col, fin.cols, v);
      if (PAIR) load_columns<COOP_F32, E>(pre2 + r * fin.cols, at.col, fin.cols, u);
      fin.slope(at, r, v, u);
    }
  }
  fin.end(at, lanes, (int64_t)blockIdx.y * kWavesPerBlock + uniform_wave_in_block());
}

// out[y][c] = sum of the y-th share of part's rows; 64 columns a block, its waves deal the rows among themselves.  Of two parts one behind the
// other (as many rows each) the second's sums are out2's.
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves* kWave) void k_dense_columns(const float* __restrict__ part, const float* __restrict__ part2, int64_t rows, int32_t cols,
                                                                    float* __restrict__ out, float* __restrict__ out2) {
  __shared__ float lds[kJoinWaves][kWave];
  if (blockIdx.z == 1) part = part2, out = out2;
  const int32_t c = (int32_t)blockIdx.x * kWave + lane_id();
  const int64_t first = rows * blockIdx.y / gridDim.y, last = rows * (blockIdx.y + 1) / gridDim.y;
  float sum = 0.f;
  if (c < cols) {
#pragma unroll 8
    for (int64_t r = first + wave_in_block(); r < last; r += kJoinWaves) sum += part[r * cols + c];
  }
  lds[wave_in_block()][lane_id()] = sum;
  __syncthreads();
  if (wave_in_block() != 0 || c >= cols) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) sum += lds[w][lane_id()];
  out[(int64_t)blockIdx.y * cols + c] = sum;
}

// Rows of `dim` elements into rows of `width`, a multiple of 16 bytes, zeros behind a row's end.  Up to four arrays in one launch.
struct Copy {
  const char* in;
  char* out;
  int64_t rows;
  int32_t dim, width;
  uint32_t first_block;
};
struct Copies {
  Copy c[4];
  int n;
};
template <int T>
__global__ __launch_bounds__(kBlock) void k_dense_pad(Copies jobs, uint32_t blocks) {
  typedef typename Element<T>::M M;
  constexpr int E = kE<T>;
  int j = 0;
  while (j + 1 < jobs.n && blockIdx.x >= jobs.c[j + 1].first_block) ++j;
  const Copy& c = jobs.c[j];
  const uint32_t end = j + 1 < jobs.n ? jobs.c[j + 1].first_block : blocks;
  const int32_t packs = c.width / E;
  for (int64_t i = (int64_t)(blockIdx.x - c.first_block) * kBlock + threadIdx.x; i < c.rows * packs; i += (int64_t)(end - c.first_block) * kBlock) {
    const int64_t row = i / packs;
    const int32_t col = (int32_t)(i - row * packs) * E;
    float f[E];
    load_columns<T, E>((const M*)c.in + row * c.dim, col, c.dim, f);
    store_elements<T, E>((M*)c.out + row * c.width + col, f);
  }
}

#include "dense_few.h"
#include "dense_narrow.h"
#include "dense_small.h"

// ---- how a call is cut ------------------------------------------------------------------------------------------------------------
// A product of rows x cols over k, in tiles of 256 x 256 (16 bits; what a wave's registers hold, a block to a CU), of 128 x 128 (two blocks) or of
// 64 x 64 (five; a pair's 64 x 128, three).  Which, by the rounds of the chip that the tiles take, and what a round takes: what a tile begins and
// ends with, which nothing hides in a block that is alone, and its stages of 128 bytes of k, which larger tiles read less of LDS for.  (bf16:
// 8,192 x 4,096 over 4,096 239 us in tiles of 256, 289 of 128; 100,000 x 768 over 128 77, 58, of 64 70; 40,000 x 512 over 1,024 72, 51, 72; 100,000
// x 64 over 768 54, 34, 29.  fp32: 50,000 x 64 over 768 98 of 128, 55 of 64.)
// k is split where there are fewer tiles than blocks that run at a time, as long as every part has four stages.  Where even so half of the chip
// would be idle the tiles are of 64: a quarter of the work for each to do one after the other.  `twice`: every stage is multiplied by both parts of B (few
// values, or few results: not in tiles of 256).
struct Cut {
  int64_t rows, cols, width;  // width: of a row of parts
  int tile_a, tile_b;
  uint32_t tiles_a, tiles_b, splits;
  size_t part_bytes;
  Cut() : rows(0), cols(0), width(0), tile_a(0), tile_b(0), tiles_a(0), tiles_b(0), splits(0), part_bytes(0) {}
  Cut(int64_t rows_, int64_t cols_, int64_t k, int dtype, bool pair, bool twice = false) : rows(rows_), cols(cols_) {
    const int per_tile = pair ? 2 : 1;
    const auto tiles_of = [&](int a, int b) { return ((cols * per_tile + a - 1) / a) * ((rows + b - 1) / b); };
    const int64_t stages = k * element_bytes(dtype) / kWide, most = stages / 4 < 1 ? 1 : stages / 4;
    const auto splits_of = [&](int a, int b) { return at_most((a == 256 ? 256 : 512) / at_most(tiles_of(a, b), 512), most); };
    // (microseconds; of splits the stages that each has, and the launch that joins them)
    const auto time_of = [&](int a, int b, int64_t slots, double ends, double stage) {
      const int64_t parts = splits_of(a, b), blocks = tiles_of(a, b) * parts;
      return (double)((blocks + slots - 1) / slots) * (ends + stage * (double)((stages < parts ? 1 : stages / parts) * (twice ? 2 : 1))) + (parts > 1 ? 6 : 0);
    };
    const bool wide = dtype == COOP_F32;
    const int small_b = pair ? 128 : 64;
    const double of_256 = time_of(256, 256, 256, 12, 1.7), of_128 = time_of(128, 128, 512, wide ? 6 : 4, wide ? 4.1 : 1.02);
    const double of_64 = time_of(64, small_b, pair ? 768 : 1280, 3, pair ? (wide ? 2.5 : 0.8) : (wide ? 2.4 : 0.95));
    tile_a = tile_b = !wide && !twice && of_256 < of_128 ? 256 : 128;
    if (tile_a == 128 && (tiles_of(128, 128) * splits_of(128, 128) <= 256 || of_64 < of_128)) tile_a = 64, tile_b = small_b;
    tiles_a = (uint32_t)((cols * per_tile + tile_a - 1) / tile_a);
    tiles_b = (uint32_t)((rows + tile_b - 1) / tile_b);
    splits = (uint32_t)splits_of(tile_a, tile_b);
    width = round_up(cols, 8) * per_tile;
    part_bytes = splits > 1 ? (size_t)splits * (size_t)rows * (size_t)width * 4 : 0;
  }
  uint64_t blocks() const { return (uint64_t)tiles_a * tiles_b * splits; }
  int64_t sum_rows(bool pair) const { return (int64_t)tiles_b * (pair && tile_a == 64 ? 4 : 2); }  // of a block's waves, those side by side along the rows
};

bool fits(const Cut& c) { return c.blocks() < ((uint64_t)1 << 31); }

bool aligned16(const void* a, const void* b, const void* c = nullptr, const void* d = nullptr) {
  return (((uintptr_t)a | (uintptr_t)b | (uintptr_t)c | (uintptr_t)d) & 15) == 0;
}
// f(KS, MT) for the steps of 16 of k and the tiles of 32 of m
template <typename F>
void with_narrow(int64_t k, int64_t m, F&& f) {
  const auto mt = [&](auto ks) {
    if (m <= 32) f(ks, std::integral_constant<int, 1>());
    else if (m <= 64) f(ks, std::integral_constant<int, 2>());
    else f(ks, std::integral_constant<int, 4>());
  };
  if (k <= 32) mt(std::integral_constant<int, 2>());
  else if (k <= 64) mt(std::integral_constant<int, 4>());
  else mt(std::integral_constant<int, 8>());
}

// whether what dz loses fits the narrow gradient's LDS
constexpr bool narrow_rest(int64_t k, int64_t m) { return k <= 32 || m <= 64; }

int narrow_shares(int64_t k, int64_t m) {
  int shares = 1;
  with_narrow(k, m, [&](auto ks, auto mt) { shares = NarrowBackward<COOP_BF16, decltype(ks)::value, decltype(mt)::value>::kShares; });
  return shares;
}

// Of 16 bits dz is an operand of the matrix units, rounded to the type, or the sum of two numbers of the type, and the products take both.  Rounded once it
// makes a gradient 1.41 times as far from 64 bits as its own rounding does, whatever the sizes, as noise of the same size does; but of few results that is 1.41 give or take
// much (worst of 8 draws, both types: 64 values of dW 2.2 times, 256 1.7, 1,024 1.6, 2,048 1.5, from 4,096 on 1.46).  So both are kept where a result, dx
// or one weight's gradient, has few values, and where dz itself has so few that it costs next to nothing.
constexpr int64_t kRestResults = 1 << 12, kRestValues = 1 << 16;

// The parts of a call, and where in the workspace they are.  GATED: two weights of m rows.
struct DensePlan {
  int64_t n, k, m, kw, mw;  // kw, mw: elements of a row of k or m, up to a multiple of 16 bytes
  int64_t dz_ld, half;      // elements; a pair's second part begins at mw, what dz loses to its type at half
  bool gated, pad, slope, again;  // slope: dz is not dout itself; again: the forward product is computed again
  bool few;                       // forward, of few rows or small: the kernel of dense_few.h
  bool small;                     // gradient, of what is small: the kernels of dense_small.h
  bool rest;                      // gradient with what dz loses to its type
  bool narrow;                    // 8 to 128 by 8 to 128 in 16 bits: the kernels of dense_narrow.h (but not from what was kept)
  uint32_t narrow_tiles, narrow_blocks;
  Cut forward, back, weight;      // (dx and dW)
  int64_t sum_rows;               // of the columns' partial sums
  int lanes_log2;
  uint32_t slope_x, slope_y, join_y;
  size_t x, w, w2, dz, pre, part, part2, join, sums, bytes;
  DensePlan(int64_t n_, int32_t k_, int32_t m_, int dtype, bool gated_, bool aligned, bool grad, bool keeps, int act) : n(n_), k(k_), m(m_), gated(gated_) {
    const int es = element_bytes(dtype), e = 16 / es;
    kw = round_up(k, e);
    mw = round_up(m, e);
    // Its blocks read, all together and mostly from L2, some times what tiles do, which need copies for alignment and a launch that joins parts; and
    // there may not be many more than run at a time.  (bf16, forward: 1,021 x 602 x 75, 9 MB: 4.1 us for 12.1; 1,024 x 1,024 x 256, 48 MB: 8.8 for
    // 10.3; 2,048 x 512 x 512, 96 MB: 13.3 both)
    const auto little = [&](int64_t blocks, int64_t rows, int64_t length, int64_t most) { return blocks <= most && blocks * rows * length * es <= 48 << 20; };
    const int64_t n_tiles = (n + kFewRows - 1) / kFewRows, k_tiles = (k + 15) / 16, both = gated ? 2 * mw : m;
    const bool few_fits = little((m + 15) / 16 * n_tiles, (gated ? 32 : 16) + kFewRows, k, (int64_t)k * es > kFewMany ? 2048 : 8192);
    few = !grad && (n <= kFewRows || few_fits);
    // (its gradient, kept products: 1,024 x 256 x 256 11.0 us for 20.5, 1,021 x 602 x 75 12.9 for 23.0, 64 x 1,024 x 1,024 16.3 for 18.4; and 2 launches
    // for 6, 3 us each to whoever launches them)
    again = grad && !keeps && (gated || act != COOP_ACT_NONE);
    small = grad && n * es <= kSmallLength && both * es <= kSmallLength && little(k_tiles * n_tiles, 16 + kSmallRows, both, 4096) &&
            little(k_tiles * ((both + kSmallRows - 1) / kSmallRows), 16 + kSmallRows, n, 4096) && (!again || few_fits);
    // (by what is computed alone, and not by which kernels do it)
    rest = grad && es == 2 && (gated || act != COOP_ACT_NONE) && (n * m * (gated ? 2 : 1) <= kRestValues || (n < m ? n : m) * k <= kRestResults);
    narrow = !few && !small && es == 2 && !gated && k >= 8 && k <= 128 && m >= 8 && m <= 128 && !(grad && keeps && act != COOP_ACT_NONE) && (!rest || narrow_rest(k, m));
    narrow_tiles = (uint32_t)((n + 31) / 32);
    narrow_blocks = (uint32_t)(grad ? at_most((narrow_tiles + 7) / 8, 256) : at_most((narrow_tiles + kNarrowForwardWaves - 1) / kNarrowForwardWaves, 512));
    pad = !narrow && !few && !small && (!aligned || kw != k);
    size_t at = 0;
    auto take = [&](size_t b) { const size_t o = at; at += (b + 255) & ~(size_t)255; return o; };
    x = take(pad ? (size_t)n * kw * es : 0);
    w = take(pad ? (size_t)m * kw * es : 0);
    w2 = take(pad && gated ? (size_t)m * kw * es : 0);
    forward = Cut(n, m, kw, dtype, gated);
    size_t parts = narrow || few ? 0 : forward.part_bytes;
    dz = pre = part = part2 = join = 0;
    slope = false;
    half = 0;
    if (grad && narrow) {
      parts = (size_t)narrow_blocks * (size_t)narrow_shares(k, m) * (size_t)m * (size_t)(round_up(k, 8) + kNarrowSums) * 4;
    } else if (grad) {
      slope = gated || act != COOP_ACT_NONE || (!small && (!aligned || mw != m));
      half = gated ? 2 * mw : mw;
      dz_ld = rest ? 2 * half : half;
      if (dz_ld * es % 2048 == 0) dz_ld += 256 / es;  // (or a tile's rows would all lie in the same few channels of memory)
      dz = take(slope ? (size_t)n * dz_ld * es : 0);
      pre = take(again && !small && forward.splits > 1 ? (size_t)n * m * 4 * (gated ? 2 : 1) : 0);
      back = Cut(n, k, mw, dtype, false, rest);
      weight = Cut(gated ? 2 * mw : m, k, n, dtype, false, rest);
      if (!again || small) parts = 0;
      if (!small && back.part_bytes > parts) parts = back.part_bytes;
      if (!small && weight.part_bytes > parts) parts = weight.part_bytes;
      // the columns' sums: by the product's waves of rows, or by the blocks that go over the rows (where they do nothing else some 1,024
      // of them: 8,192 x 4,096 bf16 18.4 us with the parts' sum; 4,096: 26.9.  With dz to write, 8,192 x 5,632 gated: 156, and 138)
      const int64_t packs = mw / e;
      lanes_log2 = 0;
      while (lanes_log2 < 6 && 1 << lanes_log2 < packs) ++lanes_log2;
      slope_x = (uint32_t)((packs + (1 << lanes_log2) - 1) >> lanes_log2);
      const int64_t groups = (n + (kBlock >> lanes_log2) - 1) / (kBlock >> lanes_log2);
      slope_y = (uint32_t)at_most(groups, small ? 128 : n * m <= 1 << 19 ? 64 : (slope ? 4096 : 1024) / slope_x + 1);  // (of little, so few that one launch adds up what they have)
      sum_rows = again && small ? (n + kSmallRows - 1) / kSmallRows * 2 : again && forward.splits == 1 ? forward.sum_rows(gated) : (int64_t)slope_y * kWavesPerBlock;
      const size_t sum_bytes = (size_t)sum_rows * (size_t)m * 4;
      part = take(sum_bytes);
      part2 = take(gated ? sum_bytes : 0);
      join_y = small || sum_rows <= 1024 ? 1 : (uint32_t)at_most(sum_rows / 256, 64);
      join = take(join_y > 1 ? (size_t)join_y * (size_t)m * 4 * (gated ? 2 : 1) : 0);
    }
    sums = take(parts);
    bytes = at;
  }
  bool fit(bool grad) const { return few || small || narrow || (fits(forward) && (!grad || (fits(back) && fits(weight)))); }
};

// Blocks of more than 64 KB of LDS have to be allowed, once for each kernel and device.
template <auto kernel>
bool allow_lds(int bytes) {
  static std::atomic<uint64_t> allowed{0};
  int device = 0;
  if (hipGetDevice(&device) != hipSuccess) return false;
  const uint64_t bit = (uint64_t)1 << (device & 63);
  if (device < 64 && (allowed.load(std::memory_order_relaxed) & bit) != 0) return true;
  if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return false;
  allowed.fetch_or(bit, std::memory_order_relaxed);
  return true;
}

template <int T, int WA, int WB, int TA, int TB, bool SA, bool SB, int SIZE, int FORM, bool TWICE, typename Fin>
bool launch_tiles(int id, const Cut& c, const Operand& a, const Operand& a2, const Operand& b, const Operand& b2, int64_t k, const Fin& fin, hipStream_t s) {
  typedef Product<T, WA, WB, TA, TB, SA, SB, SIZE, FORM == kPair> P;
  constexpr auto kernel = k_dense<T, WA, WB, TA, TB, SA, SB, SIZE, FORM, TWICE, Fin>;
  if (!allow_lds<kernel>(P::kLds)) return false;
  COOP_LAUNCH(id, kernel, dim3((unsigned)c.blocks()), dim3(P::kThreads), P::kLds, s, a, a2, b, b2, k, Tiles{c.tiles_a, c.tiles_b, c.splits}, fin);
  return true;
}
template <int T, bool SA, bool SB, int SIZE, int FORM, bool TWICE, typename Fin>
bool launch_product(int id, const Cut& c, const Operand& a, const Operand& a2, const Operand& b, const Operand& b2, int64_t k, const Fin& fin, hipStream_t s) {
  if constexpr (T != COOP_F32 && !TWICE)
    if (c.tile_a == 256) return launch_tiles<T, 2, 2, 4, 4, SA, SB, SIZE, FORM, false>(id, c, a, a2, b, b2, k, fin, s);
  if (c.tile_a == 128) return launch_tiles<T, 2, 2, 2, 2, SA, SB, SIZE, FORM, TWICE>(id, c, a, a2, b, b2, k, fin, s);
  if constexpr (FORM == kPair) return launch_tiles<T, 1, 4, 2, 1, SA, SB, SIZE, FORM, TWICE>(id, c, a, a2, b, b2, k, fin, s);  // (a wave has columns of both)
  else return launch_tiles<T, 2, 2, 1, 1, SA, SB, SIZE, FORM, TWICE>(id, c, a, a2, b, b2, k, fin, s);
}

template <int T, bool PAIR, typename Fin>
void join(const float* sums, int splits, int64_t rows, int64_t width, int32_t cols, const Fin& fin, hipStream_t s) {
  const int share = splits >= kSumWaves ? kSumWaves : 1, each = kSumWaves / share * kWave;
  const int64_t blocks = (rows * ((cols + 3) / 4) + each - 1) / each;
  COOP_LAUNCH(K_DENSE_JOIN, (k_dense_join<T, PAIR, Fin>), dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(kSumWaves * kWave), 0, s, sums, splits, share,
              rows, width, cols, fin);
}

// A product and its epilogue, through parts where k is split.
template <int T, bool SA, bool SB, int SIZE, int FORM, bool TWICE = false, typename Fin>
bool product(int id, const Cut& c, const Operand& a, const Operand& a2, const Operand& b, const Operand& b2, int64_t k, const Fin& fin, float* sums, hipStream_t s) {
  if (c.splits == 1) return launch_product<T, SA, SB, SIZE, FORM, TWICE>(id, c, a, a2, b, b2, k, fin, s);
  if (!launch_product<T, SA, SB, SIZE, FORM, TWICE>(id, c, a, a2, b, b2, k, Part<FORM == kPair>{sums, c.rows, c.width, 0}, s)) return false;
  if constexpr (!Fin::kSums) join<T, FORM == kPair>(sums, (int)c.splits, c.rows, c.width, (int32_t)c.cols, fin, s);
  return true;
}

// The same where B may have a rest (16 bits).
template <int T, bool SA, bool SB, int SIZE, int FORM, typename Fin>
bool product_of_dz(int id, const Cut& c, bool rest, const Operand& a, const Operand& a2, const Operand& b, const Operand& b2, int64_t k, const Fin& fin, float* sums,
                   hipStream_t s) {
  if constexpr (T != COOP_F32)
    if (rest) return product<T, SA, SB, SIZE, FORM, true>(id, c, a, a2, b, b2, k, fin, sums, s);
  return product<T, SA, SB, SIZE, FORM>(id, c, a, a2, b, b2, k, fin, sums, s);
}

// alpha is left to the results, so that of one below 1 no dz is lost below the numbers of its type.  (One above 1 is multiplied into dz, for the same reason: what
// falls below them is lost without a trace, and what is beyond them is an infinity that a program sees.)  Without an activation dz is dout, and all of it left to them.
struct Alpha { float into, results; };
Alpha split_alpha(float alpha, int act) {
  return act != COOP_ACT_NONE && fabsf(alpha) > 1.f ? Alpha{alpha, 1.f} : Alpha{1.f, alpha};
}

struct Arrays {  // what the products read: the caller's, or copies
  const char *x, *w, *w2;
};
template <int T>
Arrays operands(const DensePlan& p, const void* x, const void* w, const void* w2, bool want_x, char* ws, hipStream_t s) {
  if (!p.pad) return Arrays{(const char*)x, (const char*)w, (const char*)w2};
  Copies jobs;
  jobs.n = 0;
  uint32_t blocks = 0;
  const auto add = [&](const void* in, size_t at, int64_t rows) {
    const int64_t need = (rows * (p.kw / kE<T>) + kBlock - 1) / kBlock;
    jobs.c[jobs.n++] = Copy{(const char*)in, ws + at, rows, (int32_t)p.k, (int32_t)p.kw, blocks};
    blocks += (uint32_t)at_most(need, 8192);
  };
  if (want_x) add(x, p.x, p.n);
  add(w, p.w, p.m);
  if (p.gated) add(w2, p.w2, p.m);
  COOP_LAUNCH(K_DENSE_PAD, k_dense_pad<T>, dim3(blocks), dim3(kBlock), 0, s, jobs, blocks);
  return Arrays{ws + p.x, ws + p.w, ws + p.w2};
}

template <int T, bool PAIR, typename Fin>
bool forward_product(const DensePlan& p, const Arrays& o, const Fin& fin, float* sums, hipStream_t s) {
  const int64_t ld = p.kw * kElem<T>;
  Operand a{o.w, ld, p.m, ld};
  if (PAIR) a.other = o.w2 - o.w;
  const Operand b{o.x, ld, p.n, ld};
  return product<T, false, false, kWide, PAIR ? kPair : kOne>(PAIR ? K_GATED : K_LINEAR, p.forward, a, a, b, b, p.kw, fin, sums, s);
}

template <int T, bool PAIR, typename Fin>
void few_product(const DensePlan& p, const void* x, const void* w, const void* w2, const Fin& fin, hipStream_t s) {
  const bool many = p.k * kElem<T> > kFewMany, one = !Fin::kSums && p.n <= 16;
  const auto kernel = many ? (one ? k_few<T, 1, PAIR, 16, Fin> : k_few<T, 2, PAIR, 16, Fin>) : (one ? k_few<T, 1, PAIR, 4, Fin> : k_few<T, 2, PAIR, 4, Fin>);
  COOP_LAUNCH(PAIR ? K_GATED : K_LINEAR, kernel, dim3((unsigned)((p.m + 15) / 16), (unsigned)((p.n + kFewRows - 1) / kFewRows)), dim3((many ? 16 : 4) * kWave), 0, s,
              (const char*)x, (const char*)w, (const char*)w2, p.n, (int32_t)p.k, fin);
}

template <int T>
void sums_of_columns(const DensePlan& p, const float* from, const float* from2, float* db, float* db2, bool pair, char* ws, hipStream_t s) {
  int64_t rows = p.sum_rows;
  const unsigned x_blocks = (unsigned)((p.m + kWave - 1) / kWave), z = pair ? 2 : 1;
  if (p.join_y > 1) {
    float* to = (float*)(ws + p.join);
    COOP_LAUNCH(K_DENSE_COLUMNS, k_dense_columns, dim3(x_blocks, p.join_y, z), dim3(kJoinWaves * kWave), 0, s, from, from2, rows, (int32_t)p.m, to,
                to + p.join_y * p.m);
    from = to, from2 = to + p.join_y * p.m, rows = p.join_y;
  }
  COOP_LAUNCH(K_DENSE_COLUMNS, k_dense_columns, dim3(x_blocks, 1, z), dim3(kJoinWaves * kWave), 0, s, from, from2, rows, (int32_t)p.m, db, db2);
}

// a row of the narrow gradient's parts: dW's columns, and behind them the bias's
struct NarrowGradient {
  Gradient g;
  float* db;
  int32_t db_col;
  template <int E> using Lane = typename Gradient::Lane<E>;
  template <int E>
  __device__ __forceinline__ void begin(Lane<E>& l, int32_t col) const { l.col = col; }
  template <int E>
  __device__ __forceinline__ void put(Lane<E>& l, int64_t row, float (&v)[E], float (&u)[E]) const {
    if (l.col < db_col) g.put(l, row, v, u);
    else if (db != nullptr) db[row] = v[0];
  }
};

template <int T>
bool backward_narrow(const DensePlan& p, const NarrowLayer& l, const void* dout, void* dx, void* dw, int grad_dtype, float* db, char* ws, hipStream_t s) {
  bool ok = true;
  float* const sums = dw != nullptr || db != nullptr ? (float*)(ws + p.sums) : nullptr;
  const int32_t db_col = dw != nullptr ? (int32_t)round_up(p.k, 8) : 0, width = db_col + kNarrowSums;
  with_narrow(p.k, p.m, [&](auto ks, auto mt) {
    constexpr int KS = decltype(ks)::value, MT = decltype(mt)::value;
    const auto launch = [&](auto exact, auto rest) {
      constexpr auto kernel = k_narrow_grad<T, KS, MT, decltype(exact)::value, decltype(rest)::value>;
      constexpr int lds = NarrowBackward<T, KS, MT, decltype(rest)::value>::kLds;
      ok = allow_lds<kernel>(lds);
      if (ok) COOP_LAUNCH(K_DENSE_DX, kernel, dim3(p.narrow_blocks), dim3(512), lds, s, l, (const char*)dout, (char*)dx, sums, width, p.narrow_tiles);
    };
    const auto either = [&](auto rest) {
      if (p.k == KS * 16 && p.m == MT * 32 && aligned16(l.x, dout, dx)) launch(std::true_type(), rest);
      else launch(std::false_type(), rest);
    };
    if constexpr (narrow_rest(KS * 16, MT * 32))
      if (p.rest) return either(std::true_type());
    either(std::false_type());
  });
  if (!ok || sums == nullptr) return ok;
  const Gradient g{(char*)dw, nullptr, p.m, 0, (int32_t)p.k, l.results, grad_dtype};
  join<T, false>(sums, (int)p.narrow_blocks * narrow_shares(p.k, p.m), p.m, width, db_col + 1, NarrowGradient{g, db, db_col}, s);
  return true;
}

template <int T, bool PAIR>
bool forward_all(const DensePlan& p, const void* x, const void* w, const void* w2, const Forward<T, PAIR>& fin, char* ws, hipStream_t s) {
  if (p.few) {
    few_product<T, PAIR>(p, x, w, w2, fin, s);
    return true;
  }
  if constexpr (T != COOP_F32 && !PAIR)
    if (p.narrow) {
      const NarrowLayer l{(const char*)x, (const char*)w, fin.bias, p.n, (int32_t)p.k, (int32_t)p.m, fin.alpha, 1.f, fin.act};
      with_narrow(p.k, p.m, [&](auto ks, auto mt) {
        constexpr int KS = decltype(ks)::value, MT = decltype(mt)::value;
        const bool exact = p.k == KS * 16 && p.m == MT * 32 && aligned16(l.x, fin.residual, fin.out);
        const auto kernel = exact ? k_narrow<T, KS, MT, true> : k_narrow<T, KS, MT, false>;
        COOP_LAUNCH(K_LINEAR, kernel, dim3(p.narrow_blocks), dim3(kNarrowForwardWaves * kWave), 0, s, l,
                    fin.residual, fin.out, fin.pre, p.narrow_tiles);
      });
      return true;
    }
  const Arrays o = operands<T>(p, x, w, w2, true, ws, s);
  return forward_product<T, PAIR>(p, o, fin, (float*)(ws + p.sums), s);
}

template <int T, bool PAIR>
bool backward_all(const DensePlan& p, const void* dout, const void* x, const void* w, const void* w2, const void* bias, const void* bias2, const float* pre,
                  int act, float alpha, void* dx, void* dw, void* dw2, int grad_dtype, float* db, float* db2, char* ws, hipStream_t s) {
  if constexpr (T != COOP_F32 && !PAIR)
    if (p.narrow) {
      const Alpha factor = split_alpha(alpha, act);
      const NarrowLayer l{(const char*)x, (const char*)w, (const char*)bias, p.n, (int32_t)p.k, (int32_t)p.m, factor.into, factor.results, act};
      return backward_narrow<T>(p, l, dout, dx, dw, grad_dtype, db, ws, s);
    }
  const bool products = dx != nullptr || dw != nullptr;
  float* const sums = (float*)(ws + p.sums);
  Arrays o{(const char*)x, (const char*)w, (const char*)w2};
  if (!p.small && (products || p.again)) o = operands<T>(p, x, w, w2, dw != nullptr || p.again, ws, s);
  Slope<T, PAIR> fin;
  fin.bias = (const char*)bias, fin.bias2 = (const char*)bias2, fin.dout = (const char*)dout;
  fin.dz = p.slope && products ? ws + p.dz : nullptr;
  fin.part = db != nullptr || db2 != nullptr ? (float*)(ws + p.part) : nullptr;
  fin.part2 = (float*)(ws + p.part2);
  fin.rows = p.n, fin.ld = p.dz_ld, fin.second = p.mw, fin.cols = (int32_t)p.m;
  const float scale = PAIR ? 1.f : split_alpha(alpha, act).results;
  fin.alpha = alpha, fin.into = split_alpha(alpha, act).into, fin.act = act;
  fin.rest = p.rest ? p.half * kElem<T> : 0;
  if (p.again && p.small) {
    few_product<T, PAIR>(p, x, w, w2, fin, s);
  } else if (p.again && p.forward.splits == 1) {
    if (!forward_product<T, PAIR>(p, o, fin, sums, s)) return false;
  } else {
    if (p.again) {
      Forward<T, PAIR> keep{(const char*)bias, (const char*)bias2, nullptr, (float*)(ws + p.pre), (float*)(ws + p.pre) + p.n * p.m, nullptr, p.n, (int32_t)p.m, 1.f, act};
      if (!forward_product<T, PAIR>(p, o, keep, sums, s)) return false;
      pre = keep.pre;
    }
    if (fin.dz != nullptr || fin.part != nullptr)
      COOP_LAUNCH(K_DENSE_SLOPE, (k_dense_slope<T, PAIR>), dim3(p.slope_x, p.slope_y), dim3(kBlock), 0, s, pre, PAIR ? pre + p.n * p.m : nullptr, p.lanes_log2, fin);
  }
  if (p.small) {
    const int64_t ld = (p.slope ? p.dz_ld : p.m) * kElem<T>, both = PAIR ? p.mw + p.m : p.m;
    const uint32_t k_tiles = (uint32_t)((p.k + 15) / 16), n_tiles = (uint32_t)((p.n + kSmallRows - 1) / kSmallRows), m_tiles = (uint32_t)((both + kSmallRows - 1) / kSmallRows);
    const SmallGrad g{p.slope ? ws + p.dz : (const char*)dout, (const char*)x, (const char*)w, (const char*)w2, p.n, ld, p.mw, fin.rest, (int32_t)p.k, (int32_t)p.m,
                      dx != nullptr ? k_tiles * n_tiles : 0, dw != nullptr ? k_tiles * m_tiles : 0, k_tiles, fin.part, fin.part2, p.sum_rows, db, db2};
    const Gradient to_x{(char*)dx, nullptr, p.n, 0, (int32_t)p.k, scale, T}, to_w{(char*)dw, PAIR ? (char*)dw2 : nullptr, p.m, p.mw, (int32_t)p.k, scale, grad_dtype};
    const uint32_t blocks = g.dx_blocks + g.dw_blocks + (fin.part != nullptr ? (uint32_t)((p.m + kWave - 1) / kWave) * (PAIR ? 2 : 1) : 0);
    auto kernel = k_small_grad<T, PAIR, false>;
    if constexpr (T != COOP_F32)
      if (p.rest) kernel = k_small_grad<T, PAIR, true>;
    if (blocks > 0) COOP_LAUNCH(K_DENSE_DX, kernel, dim3(blocks), dim3(kSmallWaves * kWave), 0, s, g, to_x, to_w);
    return true;
  }
  if (fin.part != nullptr) sums_of_columns<T>(p, fin.part, fin.part2, db, db2, PAIR, ws, s);
  const int64_t ldk = p.kw * kElem<T>, ldz = p.slope ? p.dz_ld * kElem<T> : p.m * kElem<T>;
  const char* dz = p.slope ? ws + p.dz : (const char*)dout;
  if (dx != nullptr) {
    const Gradient g{(char*)dx, nullptr, p.n, 0, (int32_t)p.k, scale, T};
    const Operand a{o.w, ldk, ldk, p.m}, a2{o.w2, ldk, ldk, p.m};
    const Operand b{dz, ldz, p.n, p.mw * kElem<T>, fin.rest}, b2{dz + (PAIR ? p.mw * kElem<T> : 0), ldz, p.n, p.mw * kElem<T>, fin.rest};
    if (!product_of_dz<T, true, false, kWide, PAIR ? kTwo : kOne>(K_DENSE_DX, p.back, p.rest, a, a2, b, b2, p.mw, g, sums, s)) return false;
  }
  if (dw != nullptr) {
    const Gradient g{(char*)dw, PAIR ? (char*)dw2 : nullptr, p.m, p.mw, (int32_t)p.k, scale, grad_dtype};
    const Operand a{o.x, ldk, ldk, p.n}, b{dz, ldz, (PAIR ? 2 * p.mw : p.mw) * kElem<T>, p.n, fin.rest};
    if (!product_of_dz<T, true, true, kNarrow, kOne>(K_DENSE_DW, p.weight, p.rest, a, a, b, b, p.n, g, sums, s)) return false;
  }
  return true;
}

constexpr int32_t kMostWidth = 1 << 18;
constexpr int64_t kMostRows = ((int64_t)1 << 31) - 512;

bool known_act(int act) { return act == COOP_ACT_NONE || act == COOP_ACT_RELU || act == COOP_ACT_GELU || act == COOP_ACT_SILU; }

int dense_check(int64_t n, int32_t k, int32_t m, int dtype, int act) {
  if (!known_dtype(dtype) || !known_act(act)) return COOP_E_ARG;
  if (n < 0 || n > kMostRows || k < 1 || k > kMostWidth || m < 1 || m > kMostWidth) return COOP_E_ARG;
  return COOP_OK;
}
// sums over no rows
int empty_sums(void* a, int64_t a_bytes, void* b, int64_t b_bytes, hipStream_t s) {
  if (a != nullptr) clear_bytes(a, a_bytes, s);
  if (b != nullptr) clear_bytes(b, b_bytes, s);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
bool workspace_ok(const void* ws, size_t bytes, size_t need) { return need == 0 || (bytes >= need && ((uintptr_t)ws & 255) == 0); }

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" size_t coop_linear_workspace_bytes(int64_t n, int32_t k, int32_t m, int dtype, int aligned) {
  if (dense_check(n, k, m, dtype, COOP_ACT_NONE) != COOP_OK) return 0;
  return DensePlan(n, k, m, dtype, false, aligned != 0, false, false, COOP_ACT_NONE).bytes;
}

extern "C" int coop_linear(const void* x, int64_t n, int32_t k, const void* weight, int32_t m, int dtype, const void* bias, int act, float alpha,
                           const void* residual, void* out, float* pre_out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = dense_check(n, k, m, dtype, act);
  if (rc != COOP_OK) return rc;
  if (n == 0) return COOP_OK;
  if (!x || !weight || !out) return COOP_E_NULL;
  for (const void* p : {x, weight, bias, residual, (const void*)out})
    if (!aligned_for(p, dtype)) return COOP_E_ARG;
  if (((uintptr_t)pre_out & 3) != 0) return COOP_E_ARG;
  const DensePlan p(n, k, m, dtype, false, aligned16(x, weight), false, false, act);
  if (p.bytes > 0 && !workspace) return COOP_E_NULL;
  if (!p.fit(false) || !workspace_ok(workspace, workspace_bytes, p.bytes)) return COOP_E_ARG;
  bool ok = true;
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    const Forward<T, false> fin{(const char*)bias, nullptr, (const char*)residual, pre_out, nullptr, (char*)out, n, m, alpha, act};
    ok = forward_all<T, false>(p, x, weight, nullptr, fin, (char*)workspace, (hipStream_t)stream);
  });
  return ok && hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_linear_grad_workspace_bytes(int64_t n, int32_t k, int32_t m, int dtype, int act, int has_pre, int aligned) {
  if (dense_check(n, k, m, dtype, act) != COOP_OK) return 0;
  return DensePlan(n, k, m, dtype, false, aligned != 0, true, has_pre != 0, act).bytes;
}

extern "C" int coop_linear_grad(const void* dout, const void* x, int64_t n, int32_t k, const void* weight, int32_t m, int dtype, const void* bias, int act,
                                float alpha, const float* pre, void* dx, void* dweight, int grad_dtype, float* dbias, void* workspace,
                                size_t workspace_bytes, void* stream) {
  const int rc = dense_check(n, k, m, dtype, act);
  if (rc != COOP_OK) return rc;
  if (grad_dtype != COOP_F32 && grad_dtype != dtype) return COOP_E_ARG;
  if ((!dx || n == 0) && !dweight && !dbias) return COOP_OK;
  if (n > 0 && (!dout || !x || !weight)) return COOP_E_NULL;
  for (const void* p : {dout, x, weight, bias, (const void*)dx})
    if (!aligned_for(p, dtype)) return COOP_E_ARG;
  if (!aligned_for(dweight, grad_dtype) || (((uintptr_t)pre | (uintptr_t)dbias) & 3) != 0) return COOP_E_ARG;
  const DensePlan p(n, k, m, dtype, false, aligned16(x, weight, dout), true, pre != nullptr, act);
  if (p.bytes > 0 && !workspace) return COOP_E_NULL;
  if (!p.fit(true) || !workspace_ok(workspace, workspace_bytes, p.bytes)) return COOP_E_ARG;
  if (n == 0) return empty_sums(dweight, (int64_t)m * k * element_bytes(grad_dtype), dbias, (int64_t)m * 4, (hipStream_t)stream);
  bool ok = true;
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    ok = backward_all<T, false>(p, dout, x, weight, nullptr, bias, nullptr, pre, act, alpha, dx, dweight, nullptr, grad_dtype, dbias, nullptr,
                                (char*)workspace, (hipStream_t)stream);
  });
  return ok && hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_gated_workspace_bytes(int64_t n, int32_t k, int32_t f, int dtype, int aligned) {
  if (dense_check(n, k, f, dtype, COOP_ACT_NONE) != COOP_OK) return 0;
  return DensePlan(n, k, f, dtype, true, aligned != 0, false, false, COOP_ACT_NONE).bytes;
}

extern "C" int coop_gated(const void* x, int64_t n, int32_t k, const void* gate, const void* up, int32_t f, int dtype, const void* gate_bias,
                          const void* up_bias, int act, void* out, float* pre_out, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = dense_check(n, k, f, dtype, act);
  if (rc != COOP_OK) return rc;
  if (n == 0) return COOP_OK;
  if (!x || !gate || !up || !out) return COOP_E_NULL;
  for (const void* p : {x, gate, up, gate_bias, up_bias, (const void*)out})
    if (!aligned_for(p, dtype)) return COOP_E_ARG;
  if (((uintptr_t)pre_out & 3) != 0) return COOP_E_ARG;
  const DensePlan p(n, k, f, dtype, true, aligned16(x, gate, up), false, false, act);
  if (p.bytes > 0 && !workspace) return COOP_E_NULL;
  if (!p.fit(false) || !workspace_ok(workspace, workspace_bytes, p.bytes)) return COOP_E_ARG;
  bool ok = true;
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    const Forward<T, true> fin{(const char*)gate_bias, (const char*)up_bias, nullptr, pre_out, pre_out ? pre_out + n * f : nullptr, (char*)out, n, f, 1.f, act};
    ok = forward_all<T, true>(p, x, gate, up, fin, (char*)workspace, (hipStream_t)stream);
  });
  return ok && hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_gated_grad_workspace_bytes(int64_t n, int32_t k, int32_t f, int dtype, int has_pre, int aligned) {
  if (dense_check(n, k, f, dtype, COOP_ACT_NONE) != COOP_OK) return 0;
  return DensePlan(n, k, f, dtype, true, aligned != 0, true, has_pre != 0, COOP_ACT_NONE).bytes;
}

extern "C" int coop_gated_grad(const void* dout, const void* x, int64_t n, int32_t k, const void* gate, const void* up, int32_t f, int dtype,
                               const void* gate_bias, const void* up_bias, int act, const float* pre, void* dx, void* dgate, void* dup, int grad_dtype,
                               float* dgate_bias, float* dup_bias, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = dense_check(n, k, f, dtype, act);
  if (rc != COOP_OK) return rc;
  if (grad_dtype != COOP_F32 && grad_dtype != dtype) return COOP_E_ARG;
  if ((dgate == nullptr) != (dup == nullptr) || (dgate_bias == nullptr) != (dup_bias == nullptr)) return COOP_E_ARG;
  if ((!dx || n == 0) && !dgate && !dgate_bias) return COOP_OK;
  if (n > 0 && (!dout || !x || !gate || !up)) return COOP_E_NULL;
  for (const void* p : {dout, x, gate, up, gate_bias, up_bias, (const void*)dx})
    if (!aligned_for(p, dtype)) return COOP_E_ARG;
  if (!aligned_for(dgate, grad_dtype) || !aligned_for(dup, grad_dtype)) return COOP_E_ARG;
  if ((((uintptr_t)pre | (uintptr_t)dgate_bias | (uintptr_t)dup_bias) & 3) != 0) return COOP_E_ARG;
  const DensePlan p(n, k, f, dtype, true, aligned16(x, gate, up), true, pre != nullptr, act);
  if (p.bytes > 0 && !workspace) return COOP_E_NULL;
  if (!p.fit(true) || !workspace_ok(workspace, workspace_bytes, p.bytes)) return COOP_E_ARG;
  if (n == 0) {
    const int64_t bytes = (int64_t)f * k * element_bytes(grad_dtype);
    const int rc2 = empty_sums(dgate, bytes, dup, bytes, (hipStream_t)stream);
    return rc2 != COOP_OK ? rc2 : empty_sums(dgate_bias, (int64_t)f * 4, dup_bias, (int64_t)f * 4, (hipStream_t)stream);
  }
  bool ok = true;
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    ok = backward_all<T, true>(p, dout, x, gate, up, gate_bias, up_bias, pre, act, 1.f, dx, dgate, dup, grad_dtype, dgate_bias, dup_bias,
                               (char*)workspace, (hipStream_t)stream);
  });
  return ok && hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
