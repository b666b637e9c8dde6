// Softmax cross entropy over a large vocabulary without the logits kept, and its gradient.
//
// With z = alpha H W^T (H [n, dim] hidden states, W [vocab, dim]), t the rows' targets:
//   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_i,t(i),
//   G_iv = alpha dloss_i (exp(z_iv - lse_i) - [v = t(i)]),   dH = G W,   dW = G^T H.
// Forward: one product, whose tiles stay in registers and leave as a running maximum and sum per row.  Backward: the logits again, a
// piece of the vocabulary at a time, left as G of that piece in 16 bits (32 for fp32), and the two products with it.
//
// The logits are computed as vocabulary x hidden: a lane then holds many logits of one row of H, and neither maximum, sum nor target
// takes another lane until the end.
//
// Rows of up to 128 elements of 16 bits (narrow; forward, up to 256) go another way: there the exponentials weigh as much as the products,
// and G would be written and read for little arithmetic.  A wave keeps 64 rows of one operand in its registers as fragments, the other
// operand streams through LDS, and G never leaves the registers: the 32 x 32 tile of logits that a product leaves is, rounded and packed, a
// fragment of the next product, if that takes its k in the order in which the first one left its rows.  The logits are then computed three
// times (five products in the place of four), and nothing of the size of G is moved.  Backward with 256 elements the sums would not fit.
//
// Rates (2 n vocab dim for a product; a library product of 8192^3 reaches 1,382 TFLOP/s in bf16 and 153 in fp32):
//   8,192 x 232,965 x 128 bf16, narrow: statistics 525 us, 930 TFLOP/s (the matrix units at work 46% of the time; the exponentials and the
//     maximum beside them); dH, two products, 807 us, 1,210 (61%); dW 921 us, 1,060 (55%; 64 more factors a lane and stage, coef of the rows).
//   8,192 x 131,072 x 1,024 bf16: statistics 2,059 us, 1,070 (51%); G 2,427 us, 906 (45%), the 2.1 GB that it writes among it; dH 1,861, 1,180;
//     dW 1,734, 1,270.  A wave has its SIMD to itself (its sums are half of all registers): what follows a tile's products is not hidden.
//   1,021 x 50,021 x 100 fp32: 100 to 150 us each, 68 to 100 TFLOP/s: the units at work 80 to 88% of the time (G 67%), on rows taken as 128 elements.
//   24 x 232,965 x 128 bf16: 13 us, W's 60 MB at 4.5 TB/s.
#include <type_traits>

#include "coop_internal.h"
#include "dealing.h"
#include "products.h"

namespace coop {
namespace {

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
constexpr float kNoMax = -3.402823466e38f;

// Which tiles of two operands a block has, of na by nb: the 32 blocks that an XCD runs at a time have neighbouring ones, as many of b's
// as take half of its L2 (four at least) and the next few of a's, so that what the L2 takes from memory is read by several of them.
// (8,192 rows of 1,024 elements of bf16, 131,072 tokens: statistics 2,170 -> 2,059 us, and with neighbours of the same rows in the other
// two products dH 2,055 -> 1,861, dW 1,768 -> 1,734.  With a part of the vocabulary to an XCD all of H, 17 MB, was read for each tile of W.)
struct TilePair {
  uint32_t a, b;
  __device__ __forceinline__ TilePair(uint32_t na, uint32_t nb, int64_t tile_bytes) {
    if (nb == 1) {
      a = blockIdx.x, b = 0;
      return;
    }
    const uint32_t fit = (uint32_t)((2 << 20) / tile_bytes), strip = fit < 4 ? 4 : fit;
    const uint32_t i = xcd_runs(blockIdx.x, gridDim.x), first = i / (na * strip) * strip, at = i - first * na, rows = nb - first < strip ? nb - first : strip;
    a = at / rows;
    b = first + at % rows;
  }
};

// ---- forward -------------------------------------------------------------------------------------------------------------
// A block has kRowsB rows of H and every `splits`-th tile of the vocabulary; it leaves the rows' maximum, sum and target logit (all
// base 2: times log2 e) as part[split][row].
struct RowStat { float top, sum, target, pad; };

template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_stats(Operand w, Operand h, int64_t n, int64_t vocab, int64_t k, float scale2,
                                                               const int32_t* __restrict__ targets, int splits, RowStat* __restrict__ part) {
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> P;
  extern __shared__ char lds[];
  const TilePair tiles(splits, WB * TB == 1 ? 1 : gridDim.x / splits, P::kRowsB * h.ld);  // (few rows: one tile of them)
  const int split = tiles.a;
  const int64_t row0 = (int64_t)tiles.b * P::kRowsB;
  P p;
  float top[TB], sum[TB], target[TB];
  int32_t t[TB];
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int64_t i = row0 + P::b0() + j * 32 + (lane_id() & 31);
    t[j] = i < n ? targets[i] : -1;
    top[j] = kNoMax;
    sum[j] = target[j] = 0.f;
  }
  p.begin(w, h, (int64_t)split * P::kRowsA, row0, 0, k, splits * P::kRowsA, lds);
  for (int64_t v0 = (int64_t)split * P::kRowsA; v0 < vocab; v0 += (int64_t)splits * P::kRowsA) {
    p.zero();
    p.tile();
    const int first = (int)v0 + P::a0() + P::own_row(), left = (int)vocab - first;
#pragma unroll
    for (int j = 0; j < TB; ++j) {
      __builtin_amdgcn_sched_barrier(0);  // (a column of tiles at a time: all of them at once do not fit into the registers)
      const int mine = t[j] - first;
      if (ballot64((uint32_t)mine < (uint32_t)(TA * 32)) != 0) {
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (mine == i * 32 + P::row_of(e)) target[j] = p.acc[i][j][e] * scale2;
      }
      if (v0 + P::kRowsA > vocab) {  // (what is not there never is the largest, and adds nothing)
#pragma unroll
        for (int i = 0; i < TA; ++i)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (i * 32 + P::row_of(e) >= left) p.acc[i][j][e] = scale2 < 0.f ? __builtin_inff() : -__builtin_inff();
      }
      float x[TA * 16];
#pragma unroll
      for (int i = 0; i < TA; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i * 16 + e] = p.acc[i][j][e];
      // the largest times a positive factor is the largest product, rounded or not
      float m = x[0];
      if (scale2 < 0.f) {
#pragma unroll
        for (int e = 1; e < TA * 16; ++e) m = fminf(m, x[e]);
      } else {
#pragma unroll
        for (int e = 1; e < TA * 16; ++e) m = fmaxf(m, x[e]);
      }
      m = fmaxf(top[j], m * scale2);
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < TA * 16; ++e) s[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale2, -m));
      sum[j] = sum[j] * __builtin_amdgcn_exp2f(top[j] - m) + ((s[0] + s[1]) + (s[2] + s[3]));
      top[j] = m;
    }
  }
  P::end();
  // lanes l and l + 32 have the same rows, and so have the waves of a column of waves
  RowStat* stat = reinterpret_cast<RowStat*>(lds);
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const float m = fmaxf(top[j], __shfl_xor(top[j], 32, kWave));
    float s = sum[j] * __builtin_amdgcn_exp2f(top[j] - m);
    s += __shfl_xor(s, 32, kWave);
    const float tt = target[j] + __shfl_xor(target[j], 32, kWave);
    if (lane_id() < 32) stat[uniform_wave_in_block() / WB * P::kRowsB + P::b0() + j * 32 + lane_id()] = RowStat{m, s, tt, 0.f};
  }
  __syncthreads();
  for (int r = threadIdx.x; r < P::kRowsB; r += P::kThreads) {
    if (row0 + r >= n) break;
    RowStat all = stat[r];
#pragma unroll
    for (int a = 1; a < WA; ++a) {
      const RowStat x = stat[a * P::kRowsB + r];
      const float m = fmaxf(all.top, x.top);
      all.sum = all.sum * __builtin_amdgcn_exp2f(all.top - m) + x.sum * __builtin_amdgcn_exp2f(x.top - m);
      all.top = m;
      all.target += x.target;
    }
    part[(int64_t)split * n + row0 + r] = all;
  }
}

// As many lanes as a row has splits, up to a wave, join them.  (A wave for every row of 2.4 million, one split each: 589 us.)
__global__ __launch_bounds__(kBlock) void k_xent_loss(const RowStat* __restrict__ part, int splits, int lanes_log2, int64_t n, int64_t vocab,
                                                      const int32_t* __restrict__ targets, int32_t ignore, float* __restrict__ loss,
                                                      float* __restrict__ lse, int32_t* __restrict__ bad) {
  const int lanes = 1 << lanes_log2, lane = lane_id() & (lanes - 1);
  const int64_t i = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> lanes_log2;
  if (i >= n) return;
  float m = kNoMax, sum = 0.f, target = 0.f;
  for (int s = lane; s < splits; s += lanes) {
    const RowStat x = part[s * n + i];
    const float top = fmaxf(m, x.top);
    sum = sum * __builtin_amdgcn_exp2f(m - top) + x.sum * __builtin_amdgcn_exp2f(x.top - top);
    m = top;
    target += x.target;
  }
  for (int off = 1; off < lanes; off <<= 1) {
    const float top = fmaxf(m, __shfl_xor(m, off, kWave)), mine = sum * __builtin_amdgcn_exp2f(m - top);
    sum = mine + __shfl_xor(mine, off, kWave);
    target += __shfl_xor(target, off, kWave);
    m = top;
  }
  if (lane != 0) return;
  const int32_t t = targets[i];
  const bool ok = t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab;
  if (!ok && t != ignore) atomicOr(bad, 1);
  const float l = log2f(sum);
  lse[i] = (m + l) * kLn2;
  loss[i] = ok ? ((m - target) + l) * kLn2 : 0.f;
}

// ---- backward ------------------------------------------------------------------------------------------------------------
// What the rows of G need, all of them filled up to a multiple of a tile; target -1: the row has none, coef is 0, and its hidden state is
// taken as zeros whatever it holds.  undo (null: 1): what the row's coef is to be multiplied by, a power of two.
struct RowTerms { float *coef, *lse2; int32_t* target; float* undo; };

// G is an operand of the matrix units and has their 16 bits: the gradients are off by 1.96e-3 where exact ones rounded to bf16 are by 1.66e-3
// (fp16 2.9e-4 and 2.5e-4), all of it G's rounding; held as two operands it would double the products with it.
// In 16 bits G holds coef over the largest |coef| (and times 2^13 in fp16, whose exponents would otherwise not reach from 1 to a
// probability times dloss): where all rows count alike, as in a mean, the factor is 1 (a power of two), and so a target's p - 1 of a
// small p is not rounded away from -1 twice; with dloss itself in G, dH and dW of the mean were off by 3.0e-3 instead of 2.0e-3 (bf16).
// G in memory in fp16: a coef below 2^-10 of the largest is lifted above that by a power of two, or its row's probabilities would be lost
// below fp16's least numbers (131,072 vertices, 136 elements, rows of 1e-6 of the largest dloss: their dH off by 4e-3 to 5e-3, of 1e-7 by
// 4e-2; lifted by 3e-4 to 5e-4, as the other rows').  dH's row gets the power back when it is rounded; G's own ahead of the product for dW,
// whose sums over the rows have one scale: a launch of 2 us where no row was lifted, 70 of 1,040 us where half of them were (4,096 rows,
// 50,257 vertices, 768 elements).
constexpr int kLeast = 10;
template <int T>
constexpr float kLift = T == COOP_F16 ? 13.f : 0.f;
template <int T>
constexpr float kOne = T == COOP_F16 ? 8192.f : 1.f;

// the largest among a block's 1024 threads
__device__ __forceinline__ float block_max(float top) {
  __shared__ float lds[16];
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
  if (lane_id() == 0) lds[wave_in_block()] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 16; ++w) top = fmaxf(top, lds[w]);
  return top;
}
// the largest |coef| among a thread's rows first, first + step, .. that count
__device__ __forceinline__ float rows_top(const int32_t* __restrict__ targets, int32_t ignore, const float* __restrict__ dloss, float alpha,
                                          int64_t first, int64_t step, int64_t n, int64_t vocab) {
  float top = 0.f;
  for (int64_t i = first; i < n; i += step) {
    const int32_t t = targets[i];
    const float c = fabsf(alpha * dloss[i]);
    if (t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab && c < __builtin_inff()) top = fmaxf(top, c);
  }
  return top;
}

// Up to kTopRows rows every block of k_xent_terms looks for the largest itself, which costs less than a launch; of more rows, up to 256
// blocks do, and it looks through theirs.
constexpr int64_t kTopRows = 32768;
__global__ __launch_bounds__(1024) void k_xent_top(const int32_t* __restrict__ targets, int32_t ignore, const float* __restrict__ dloss, float alpha,
                                                   int64_t n, int64_t vocab, float* __restrict__ tops) {
  const float top = block_max(rows_top(targets, ignore, dloss, alpha, (int64_t)blockIdx.x * 1024 + threadIdx.x, (int64_t)gridDim.x * 1024, n, vocab));
  if (threadIdx.x == 0) tops[blockIdx.x] = top;
}

template <bool LIFT>
__global__ __launch_bounds__(1024) void k_xent_terms(const int32_t* __restrict__ targets, int32_t ignore, const float* __restrict__ lse,
                                                     const float* __restrict__ dloss, float alpha, float most, int64_t n, int64_t rows, int64_t vocab,
                                                     const float* __restrict__ tops, int n_tops, RowTerms term, float* __restrict__ unlift, int32_t* __restrict__ bad) {
  float top = 0.f;
  if constexpr (LIFT) {
    if (n_tops == 0) top = rows_top(targets, ignore, dloss, alpha, threadIdx.x, 1024, n, vocab);
    else if ((int)threadIdx.x < n_tops) top = tops[threadIdx.x];
    top = block_max(top);
    if (top < 0x1p-100f) top = 0x1p-100f;
    if (top > 0x1p100f) top = 0x1p100f;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *unlift = LIFT ? top / most : 1.f;
  const int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x;
  if (i >= rows) return;
  float coef = 0.f, lse2 = 0.f, undo = 1.f;
  int32_t target = -1;
  if (i < n) {
    const int32_t t = targets[i];
    if (t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab) {
      const float part = LIFT ? alpha * dloss[i] / top : alpha * dloss[i];
      coef = LIFT ? part * most : part;
      if (term.undo != nullptr) {
        const int below = 127 - (int)(__float_as_uint(part) >> 23 & 0xFFu) - kLeast;  // (at most 117; a NaN's or an infinity's is negative)
        if (below > 0 && part != 0.f) {
          undo = __uint_as_float((uint32_t)(127 - below) << 23);
          coef *= __uint_as_float((uint32_t)(127 + below) << 23);
        }
      }
      lse2 = lse[i] * kLog2e;
      target = t;
    } else if (t != ignore) {
      atomicOr(bad, 1);
    }
  }
  term.coef[i] = coef;
  term.lse2[i] = lse2;
  term.target[i] = target;
  if (term.undo != nullptr) term.undo[i] = undo;
}

template <int T>
__device__ __forceinline__ void put4(char* p, const float (&f)[4]) {
  Pack<T, 4> x;
  x.set(f);
  x.store(p);
}

// columns c .. c + 3 of a row of `dim`, those that there are
template <int T>
__device__ __forceinline__ void put_columns(char* out, int64_t row, int64_t c, int32_t dim, const float (&f)[4]) {
  char* to = out + (row * dim + c) * kElem<T>;
  if (c + 4 <= dim) {
    put4<T>(to, f);
  } else if (c < dim) {  // (one to three)
    typename Element<T>::M* at = (typename Element<T>::M*)to;
    at[0] = (typename Element<T>::M)f[0];
    if (c + 1 < dim) at[1] = (typename Element<T>::M)f[1];
    if (c + 2 < dim) at[2] = (typename Element<T>::M)f[2];
  }
}

// G of the piece of the vocabulary that begins at v_first, [rows of H, ld bytes]; all of G's tiles are there, beyond the vocabulary's
// and the rows' end it is zero.  A tile a block: its stores to G, which take a quarter of its time (128 KB a CU), go on while the next
// block is at its products.  (Blocks that went from tile to tile waited for them behind their next loads: 677 us a piece of 512 MB, 630 so.)
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_g(Operand w, Operand h, int64_t vocab, int64_t k, float scale2, int64_t v_first,
                                                           uint32_t tiles_a, RowTerms term, char* __restrict__ g, int64_t ld) {
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> P;
  extern __shared__ char lds[];
  const TilePair tiles(tiles_a, WB * TB == 1 ? 1 : gridDim.x / tiles_a, P::kRowsB * h.ld);
  const int64_t piece0 = (int64_t)tiles.a * P::kRowsA, row0 = (int64_t)tiles.b * P::kRowsB;
  P p;
  p.begin(w, h, v_first + piece0, row0, 0, k, 0, lds);
  p.zero();
  p.tile();
  P::end();
  const int first = (int)(v_first + piece0) + P::a0() + P::own_row(), left = (int)vocab - first;
  const bool ragged = v_first + piece0 + P::kRowsA > vocab;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t i = row0 + P::b0() + j * 32 + (lane_id() & 31);
    const float coef = term.coef[i], lse2 = term.lse2[i];
    const int mine = term.target[i] - first;
    const bool hit = ballot64(mine >= 0 && mine < TA * 32) != 0;
    char* to = g + i * ld + (piece0 + P::a0() + P::own_row()) * kElem<T>;
#pragma unroll
    for (int a = 0; a < TA; ++a) {
      f32x16 x = p.acc[a][j];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale2, -lse2));
      if (hit) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (mine == a * 32 + P::row_of(e)) x[e] -= 1.f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] *= coef;
      if (ragged) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (a * 32 + P::row_of(e) >= left) x[e] = 0.f;
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f[4] = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
        put4<T>(to + (a * 32 + P::row_of(4 * q)) * kElem<T>, f);
      }
    }
  }
}

// The powers of two that G's rows (fp16) were lifted by taken back: 64 rows a block, most of which have none, blockIdx.y for parts of their
// columns.
__global__ __launch_bounds__(kBlock) void k_xent_lower(const float* __restrict__ undo, int64_t n, int64_t bytes, int64_t ld, char* __restrict__ g) {
  const int64_t row0 = (int64_t)blockIdx.x * kWave;
  const float mine = row0 + lane_id() < n ? undo[row0 + lane_id()] : 1.f;
  for (uint64_t left = ballot64(mine != 1.f); left != 0; left &= left - 1) {
    const int r = __builtin_ctzll(left);
    const float u = __shfl(mine, r, kWave);
    for (int64_t at = ((int64_t)blockIdx.y * kBlock + threadIdx.x) * 16; at < bytes; at += (int64_t)gridDim.y * (kBlock * 16)) {
      char* p = g + (row0 + r) * ld + at;
      float f[8];
      load_elements<COOP_F16, 8>(p, f);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] *= u;
      store_elements<COOP_F16, 8>(p, f);
    }
  }
}

// dH: sums[split][row][dim] (+)= the split's part of G W over the piece
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_dh(Operand wt, Operand g, int64_t k, int splits, uint32_t tiles_a, uint32_t tiles_b,
                                                            bool add, float* __restrict__ sums, int64_t width) {
  typedef Product<T, WA, WB, TA, TB, true, false, kWide> P;
  extern __shared__ char lds[];
  // (neighbours have the same rows of G and another part of W's columns)
  const uint32_t i = xcd_runs(blockIdx.x, gridDim.x), tile = i / tiles_a, split = tile % splits;
  const int64_t col0 = (int64_t)(i % tiles_a) * P::kRowsA, row0 = (int64_t)(tile / splits) * P::kRowsB;
  const int64_t stages = (k + P::kK - 1) / P::kK;
  const int64_t k0 = stages * split / splits * P::kK, k1 = stages * (split + 1) / splits * P::kK;
  P p;
  p.begin(wt, g, col0, row0, k0, k1, 0, lds);
  float* to = sums + ((int64_t)split * tiles_b * P::kRowsB + row0 + P::b0() + (lane_id() & 31)) * width;
  const int c0 = (int)col0 + P::a0() + P::own_row();
  p.zero();
  if (add) {  // (the pieces' sums before this one are what it adds to)
#pragma unroll
    for (int j = 0; j < TB; ++j)
#pragma unroll
      for (int a = 0; a < TA; ++a)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = c0 + a * 32 + P::row_of(4 * q);
          if (c >= width) continue;
          float f[4];
          load_elements<COOP_F32, 4>(to + (int64_t)j * 32 * width + c, f);
#pragma unroll
          for (int e = 0; e < 4; ++e) p.acc[a][j][4 * q + e] = f[e];
        }
  }
  p.tile();
  P::end();
#pragma unroll
  for (int j = 0; j < TB; ++j)
#pragma unroll
    for (int a = 0; a < TA; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int c = c0 + a * 32 + P::row_of(4 * q);
        if (c >= width) continue;
        const float f[4] = {p.acc[a][j][4 * q], p.acc[a][j][4 * q + 1], p.acc[a][j][4 * q + 2], p.acc[a][j][4 * q + 3]};
        store_elements<COOP_F32, 4>(to + (int64_t)j * 32 * width + c, f);
      }
}

// out[row, :] = the splits' sums of the row, times *unlift and (not null) undo[row].  A wave has 64 packs of four columns; where there are many splits the block's
// waves deal those of the same packs among themselves (`share` of them), and the first adds up what they have, in their order.
constexpr int kOutWaves = 8;
template <int T>
__global__ __launch_bounds__(kOutWaves* kWave) void k_xent_out(const float* __restrict__ sums, int splits, int share, int64_t rows, int32_t width,
                                                               int64_t n, int32_t dim, const float* __restrict__ unlift, const float* __restrict__ undo,
                                                               char* __restrict__ out) {
  __shared__ float lds[4][kOutWaves][kWave];
  const int32_t packs = (dim + 3) / 4;
  const float u = *unlift;
  const int wave = uniform_wave_in_block(), lane = lane_id(), mine = wave % share, each = kOutWaves / share * kWave;
  for (int64_t first = (int64_t)blockIdx.x * each; first < n * packs; first += (int64_t)gridDim.x * each) {
    const int64_t i = first + wave / share * kWave + lane, row = i / packs;
    const int32_t c = (int32_t)(i - row * packs) * 4;
    const bool live = row < n;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (live) {
#pragma unroll 4
      for (int q = mine; q < splits; q += share) {
        float f[4];
        load_elements<COOP_F32, 4>(sums + ((int64_t)q * rows + row) * width + c, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += f[e];
      }
    }
    if (share > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < 4; ++e) lds[e][wave][lane] = s[e];
      __syncthreads();
    }
    if (mine != 0 || !live) continue;
    for (int w = 1; w < share; ++w)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] += lds[e][wave + w][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] *= u;
    if (undo != nullptr) {
      const float back = undo[row];
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] *= back;
    }
    put_columns<T>(out, row, c, dim, s);
  }
}

// dW of the piece, rows v_first .. of the weight's gradient: to out, or, split over H's rows, to sums[split][row of the piece][width].
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_dw(
    Operand ht, Operand gt, int64_t k, int splits, int64_t vocab, int64_t v_first, int32_t dim, uint32_t tiles_a, const float* __restrict__ unlift,
    char* __restrict__ out, float* __restrict__ sums, int64_t rows, int64_t width) {
  typedef Product<T, WA, WB, TA, TB, true, true, kNarrow> P;
  extern __shared__ char lds[];
  const uint32_t i = xcd_runs(blockIdx.x, gridDim.x), tile = i / tiles_a, split = tile % splits;  // (as in k_xent_dh)
  const int64_t col0 = (int64_t)(i % tiles_a) * P::kRowsA, piece0 = (int64_t)(tile / splits) * P::kRowsB;
  const int64_t stages = (k + P::kK - 1) / P::kK;
  P p;
  p.begin(ht, gt, col0, piece0, stages * split / splits * P::kK, stages * (split + 1) / splits * P::kK, 0, lds);
  p.zero();
  p.tile();
  P::end();
  const float u = *unlift;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int64_t at = piece0 + P::b0() + j * 32 + (lane_id() & 31), v = v_first + at;
    if (v >= vocab) continue;
#pragma unroll
    for (int a = 0; a < TA; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t c = col0 + P::a0() + P::own_row() + a * 32 + P::row_of(4 * q);
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = sums == nullptr ? p.acc[a][j][4 * q + e] * u : p.acc[a][j][4 * q + e];
        if (sums == nullptr) put_columns<T>(out, v, c, dim, f);
        else if (c < width) store_elements<COOP_F32, 4>(sums + ((int64_t)split * rows + at) * width + c, f);
      }
  }
}

// ---- narrow: rows of up to 128 (forward 256) elements of 16 bits -----------------------------------------------------------------------------
// A stage: 64 rows of 16 KS elements, in LDS as their chunks of 16 bytes, exchanged by the row's number: what 8 or 16 lanes read of one
// chunk of successive rows lies in different banks, and so does what they read of four rows' same 16 elements (transposed).
template <int T, int KS>
struct RowStage {
  static constexpr int kRows = 64, kRowBytes = KS * 32, kChunks = KS * 2, kBytes = kRows * kRowBytes, kMine = kBytes / 4096;
  static __device__ __forceinline__ int swizzle(int row) {
    const int r0 = row & 1, r1 = row >> 1 & 1, r2 = row >> 2 & 1, r3 = row >> 3 & 1;
    return KS == 16 ? r2 | r0 << 1 | r1 << 2 : KS == 8 ? r2 | r0 << 1 | r1 << 2 | r3 << 3 : KS == 4 ? r2 | (r0 ^ r3) << 1 | r1 << 2 : r2 | (r1 ^ r3) << 1;
  }
  // A lane's places in what it reads (from step to step and tile to tile they are an exclusive or with a few bits) and in what it loads:
  // 16 bytes of a row, the other loads of a stage in the same chunk as many rows further on.
  struct Places {
    uint32_t rows, across;
    int load;
    __device__ __forceinline__ Places() {}
    __device__ __forceinline__ Places(int wave, int lane, int ld) {
      const int r = lane & 31, b = lane >> 4, t = lane & 15, q = (b >> 1) * 4 + (t >> 2), c = (b & 1) * 16 + (t & 3) * 4;
      rows = (uint32_t)(r * kRowBytes + (((lane >> 5) ^ swizzle(r)) << 4));
      across = (uint32_t)(q * kRowBytes + (((c >> 3) ^ swizzle(q)) << 4) + (c & 7) * 2);
      const int place = wave * kWave + lane, row = place / kChunks, chunk = (place % kChunks) ^ swizzle(row);
      static_assert(4096 / kRowBytes % (KS == 16 ? 8 : 16) == 0, "the exchange of chunks goes by the row's last three or four bits");
      load = chunk * 16 < ld ? row * ld + chunk * 16 : 0x3FFFFFFF;
    }
  };
  // rows block * 32 + .., elements kk * 16 + ..: a fragment with the elements as k
  static __device__ __forceinline__ u32x4 fragment(const char* lds, uint32_t rows, int block, int kk) {
    return *reinterpret_cast<const u32x4*>(lds + (rows ^ (uint32_t)(kk << 5)) + block * 32 * kRowBytes);
  }
  // elements tile * 32 + .., with 16 of the block's rows as k, in the order in which a lane's registers hold the rows of a product
  static __device__ __forceinline__ u32x4 transposed(const char* lds, uint32_t across, int block, int tile, int s) {
    u32x4 f;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const char* from = lds + (across ^ (uint32_t)((tile << 6) ^ ((swizzle(q * 8) & (kChunks - 1)) << 4))) + (block * 32 + s * 16 + q * 8) * kRowBytes;
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(LdsByte*)from));
      f[2 * q] = y[0];
      f[2 * q + 1] = y[1];
    }
    return f;
  }
};

// lane_id(), of which the compiler does not know that it stays the same: what is made of it is made again where it is used, and not kept
__device__ __forceinline__ int lane_anew() {
  uint32_t none = 0;
#ifdef __HIP_DEVICE_COMPILE__
  asm volatile("" : "+s"(none));
#endif
  return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, none));
}

// The stages of rows first, first + step, .. of an operand, four in LDS (two of 32 KB); with TERMS the rows' coef, lse2 and target go with
// them.  Four waves.  SUMS: the waves keep sums beside their rows, and there are no registers for the lanes' places: they lie in LDS, and are
// read each stage.  (Spilled, a wait for them would be a wait for the loads of the stages ahead; made anew they cost 4% of dW's time.)
template <int T, int KS, bool TERMS, bool SUMS>
struct RowStream {
  typedef RowStage<T, KS> S;
  static constexpr int kStages = KS == 16 ? 2 : 4, kStage = S::kBytes + (TERMS ? 1024 : 0), kLds = kStages * kStage + (SUMS ? 4096 : 0), kLoads = S::kMine + (TERMS ? 1 : 0);
  const char* base;   // of the next stage
  const char* terms;  // of its rows: a wave has one of the three arrays (the last one the first again: all waves have as many loads)
  int left, step;     // rows that there are from the next stage's first (or less than none); from stage to stage
  int ld, wave, slot;
  typename S::Places kept;
  char* lds;
  __device__ __forceinline__ u32x4* mine() const { return reinterpret_cast<u32x4*>(lds + kStages * kStage) + wave * kWave + lane_anew(); }
  __device__ __forceinline__ void start(char* __restrict__ into, int at) {
#pragma unroll
    for (int i = 0; i < S::kMine; ++i) {  // (a buffer for each: the places further on would take registers that there are not)
      const int skip = i * (4096 / S::kRowBytes), there = left < S::kRows ? left - skip : S::kRows - skip;
      const int bytes = __builtin_amdgcn_readfirstlane(there > 0 ? there * ld : 0);
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(base + skip * ld), 0, bytes, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (__attribute__((address_space(3))) void*)(LdsByte*)(into + (i * 4 + wave) * 1024), 16, at, 0, 0, 0);
    }
    if constexpr (TERMS) {  // (arrays padded to 256 rows)
      const auto tr = __builtin_amdgcn_make_buffer_rsrc((void*)terms, 0, left > 0 ? S::kRows * 4 : 0, 0x00020000);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(tr, (__attribute__((address_space(3))) void*)(LdsByte*)(into + S::kBytes + (wave == 3 ? 0 : wave) * 256), 4,
                                               lane_anew() * 4, 0, 0, 0);
      terms += (int64_t)step * 4;
    }
    base += (int64_t)step * ld;
    left -= step;
  }
  __device__ __forceinline__ RowStream(const Operand& op, int first, int step_, const RowTerms* t, char* lds_)
      : left((int)op.rows - first), step(step_), ld((int)op.ld), wave(uniform_wave_in_block()), lds(lds_) {
    base = op.base + (int64_t)first * ld;
    if constexpr (TERMS) terms = (wave == 1 ? (const char*)t->coef : wave == 2 ? (const char*)t->target : (const char*)t->lse2) + (int64_t)first * 4;
    const typename S::Places places(wave, lane_id(), ld);
    if constexpr (SUMS) *mine() = u32x4{places.rows, places.across, (uint32_t)places.load, 0u};
    else kept = places;
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) start(lds + s * kStage, places.load);
    slot = kStages - 1;
  }
  static __device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * kLoads) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  // f(stage, places) for the next stage, while another one is loaded into the place of the one before it
  template <typename F>
  __device__ __forceinline__ void stage(F&& f) {
    const int from = slot + 1 < kStages ? slot + 1 : 0;
    meet();
    if constexpr (SUMS) {
      const u32x4 x = *mine();
      kept.rows = x[0], kept.across = x[1], kept.load = (int)x[2];
    }
    both(lds + slot * kStage, lds + from * kStage, f);
    slot = from;
  }
  template <typename F>
  __device__ __forceinline__ void both(char* __restrict__ into, const char* __restrict__ from, F&& f) {
    start(into, kept.load);
    f(from, kept);
  }
};

// the fragments of 64 rows of an operand that a wave keeps: rows row0 + j * 32 + .. (zeros where there are none; loads of a buffer, since
// behind a branch each would be waited for by itself)
template <int KS>
__device__ __forceinline__ void keep_rows(const Operand& op, int64_t row0, u32x4 (&x)[2][KS]) {
  const int64_t there = op.rows - row0;
  const int rows = there < 0 ? 0 : there < 64 ? (int)there : 64, ld = (int)op.ld;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(op.base + (there > 0 ? row0 : 0) * ld), 0, rows * ld, 0x00020000);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int kk = 0; kk < KS; ++kk) {
      const int at = kk * 32 + (lane_id() >> 5) * 16;
      x[j][kk] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at < ld ? (j * 32 + (lane_id() & 31)) * ld + at : 0x3FFFFFFF, 0, 0);
    }
}
__device__ __forceinline__ constexpr int row_of(int e) { return (e >> 2) * 8 + (e & 3); }  // (as in Product)
__device__ __forceinline__ int own_row() { return (lane_id() >> 5) * 4; }

// 16 values as two fragments: elements 0 .. 7 and 8 .. 15
template <int T>
__device__ __forceinline__ void pack(const f32x16& x, u32x4 (&f)[2]) {
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    Pack<T, 8> p;
#pragma unroll
    for (int e = 0; e < 8; ++e) p.x[e] = (typename Element<T>::M)x[s * 8 + e];
    f[s] = __builtin_bit_cast(u32x4, p);
  }
}

// Forward: as k_xent_stats; a block has 256 rows of H, a wave 64 of them, and every splits-th stage of 64 rows of W.  (10,784 rows, 11,256
// vertices, 256 elements of bf16: 70 us; in tiles of 256 x 256, whose exponentials nothing hides, 121.)
template <int T, int KS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_xent_stats_narrow(
    Operand w, Operand h, int64_t n, int64_t vocab, float scale2, const int32_t* __restrict__ targets, int splits, RowStat* __restrict__ part) {
  typedef RowStream<T, KS, false, false> Stream;
  typedef typename Stream::S S;
  extern __shared__ char lds[];
  const int split = blockIdx.x % splits;
  const int64_t row0 = (int64_t)(blockIdx.x / splits) * 256 + uniform_wave_in_block() * 64;
  u32x4 hf[2][KS];
  keep_rows<KS>(h, row0, hf);
  float top[2], sum[2], target[2];
  int32_t t[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t i = row0 + j * 32 + (lane_id() & 31);
    t[j] = i < n ? targets[i] : -1;
    top[j] = kNoMax;
    sum[j] = target[j] = 0.f;
  }
  Stream stream(w, split * S::kRows, splits * S::kRows, nullptr, lds);
  for (int left = (int)vocab - split * S::kRows; left > 0; left -= splits * S::kRows) {
    const int v0 = (int)vocab - left;
    f32x16 z[2][2];
    stream.stage([&](const char* from, const typename S::Places& at) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[b][0][e] = z[b][1][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          const u32x4 a = S::fragment(from, at.rows, b, kk);
#pragma unroll
          for (int j = 0; j < 2; ++j) z[b][j] = mma<T>(a, hf[j][kk], z[b][j]);
        }
      }
    });
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int mine = t[j] - v0 - own_row();
      if (ballot64((uint32_t)mine < 64u) != 0) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (mine == b * 32 + row_of(e)) target[j] = z[b][j][e] * scale2;
      }
      if (left < S::kRows) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if (b * 32 + row_of(e) + own_row() >= left) z[b][j][e] = scale2 < 0.f ? __builtin_inff() : -__builtin_inff();
      }
      float m = z[0][j][0];
      if (scale2 < 0.f) {
#pragma unroll
        for (int e = 1; e < 32; ++e) m = fminf(m, z[e >> 4][j][e & 15]);
      } else {
#pragma unroll
        for (int e = 1; e < 32; ++e) m = fmaxf(m, z[e >> 4][j][e & 15]);
      }
      m = fmaxf(top[j], m * scale2);
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 32; ++e) s[e & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(z[e >> 4][j][e & 15], scale2, -m));
      sum[j] = sum[j] * __builtin_amdgcn_exp2f(top[j] - m) + ((s[0] + s[1]) + (s[2] + s[3]));
      top[j] = m;
    }
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {  // lanes l and l + 32 have the same row
    const float m = fmaxf(top[j], __shfl_xor(top[j], 32, kWave));
    float s = sum[j] * __builtin_amdgcn_exp2f(top[j] - m);
    s += __shfl_xor(s, 32, kWave);
    const float tt = target[j] + __shfl_xor(target[j], 32, kWave);
    const int64_t i = row0 + j * 32 + lane_id();
    if (lane_id() < 32 && i < n) part[(int64_t)split * n + i] = RowStat{m, s, tt, 0.f};
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // (no load into LDS is left when the block ends)
}

// dH: sums[split][row][width] = the split's part of G W; rows, splits and stages as in the forward kernel.  A row's coef waits for the end,
// where it is one product for a sum: what is rounded to 16 bits is p itself, the target's less 1 (in fp16 times 2^13, as G below).
template <int T, int KS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_xent_dh_narrow(
    Operand w, Operand h, int64_t rows, int64_t vocab, float scale2, RowTerms term, int splits, float* __restrict__ sums, int32_t width) {
  typedef RowStream<T, KS, false, true> Stream;
  typedef typename Stream::S S;
  extern __shared__ char lds[];
  const int split = blockIdx.x % splits;
  const int64_t row0 = (int64_t)(blockIdx.x / splits) * 256 + uniform_wave_in_block() * 64;
  u32x4 hf[2][KS];
  keep_rows<KS>(h, row0, hf);
  float lse2[2];
  int32_t t[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t i = row0 + j * 32 + (lane_id() & 31);
    lse2[j] = term.lse2[i] - kLift<T>, t[j] = term.target[i] - own_row();
  }
  f32x16 acc[KS / 2][2];
#pragma unroll
  for (int c = 0; c < KS / 2; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][0][e] = acc[c][1][e] = 0.f;
  Stream stream(w, split * S::kRows, splits * S::kRows, nullptr, lds);
  for (int left = (int)vocab - split * S::kRows; left > 0; left -= splits * S::kRows) {
    const int v0 = (int)vocab - left;
    stream.stage([&](const char* from, const typename S::Places& at) {
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        f32x16 z[2];
        u32x4 p[2][2];
#pragma unroll
        for (int e = 0; e < 16; ++e) z[0][e] = z[1][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          const u32x4 a = S::fragment(from, at.rows, b, kk);
#pragma unroll
          for (int j = 0; j < 2; ++j) z[j] = mma<T>(a, hf[j][kk], z[j]);
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
#pragma unroll
          for (int e = 0; e < 16; ++e) z[j][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][e], scale2, -lse2[j]));
          const int mine = t[j] - v0 - b * 32;
          if (ballot64((uint32_t)mine < 32u) != 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (mine == row_of(e)) z[j][e] -= kOne<T>;
          }
          if (left < S::kRows) {  // (rows of W that are not there are zeros in the next product, but an exponential may be infinite)
            const int own = (lane_anew() >> 5) * 4;
#pragma unroll
            for (int e = 0; e < 16; ++e)
              if (row_of(e) + own >= left - b * 32) z[j][e] = 0.f;
          }
          pack<T>(z[j], p[j]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int c = 0; c < KS / 2; ++c) {
            const u32x4 a = S::transposed(from, at.across, b, c, s);
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[c][j] = mma<T>(a, p[j][s], acc[c][j]);
          }
      }
    });
  }
  const int lane = lane_anew(), own = (lane >> 5) * 4;
  float coef[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) coef[j] = term.coef[row0 + j * 32 + (lane & 31)] / kOne<T>;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int64_t i = row0 + j * 32 + (lane & 31);
    float* to = sums + ((int64_t)split * rows + i) * width;
#pragma unroll
    for (int c = 0; c < KS / 2; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = c * 32 + row_of(4 * q) + own;
        const float f[4] = {acc[c][j][4 * q] * coef[j], acc[c][j][4 * q + 1] * coef[j], acc[c][j][4 * q + 2] * coef[j], acc[c][j][4 * q + 3] * coef[j]};
        if (col < width) put4<COOP_F32>((char*)(to + col), f);
      }
  }
}

// dW: a block has 256 rows of W, a wave 64 of them, and every splits-th stage of 64 rows of H with their terms; to out, or, split, to
// sums[split][row][width].
template <int T, int KS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_xent_dw_narrow(
    Operand w, Operand h, int64_t vocab, float scale2, RowTerms term, int splits, const float* __restrict__ unlift, int32_t dim,
    char* __restrict__ out, float* __restrict__ sums, int64_t rows, int32_t width) {
  typedef RowStream<T, KS, true, true> Stream;
  typedef typename Stream::S S;
  extern __shared__ char lds[];
  const int split = blockIdx.x % splits;
  const int64_t v0 = (int64_t)(blockIdx.x / splits) * 256 + uniform_wave_in_block() * 64;
  u32x4 wf[2][KS];
  keep_rows<KS>(w, v0, wf);
  f32x16 acc[KS / 2][2];
#pragma unroll
  for (int c = 0; c < KS / 2; ++c)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[c][0][e] = acc[c][1][e] = 0.f;
  Stream stream(h, split * S::kRows, splits * S::kRows, &term, lds);
  for (int left = (int)h.rows - split * S::kRows; left > 0; left -= splits * S::kRows) {
    stream.stage([&](const char* from, const typename S::Places& at) {
      const int lane = lane_anew(), own = (lane >> 5) * 4;
      const float* lse2 = reinterpret_cast<const float*>(from + S::kBytes);
      const float* coef = lse2 + 64;
      const uint64_t hits = ballot64(reinterpret_cast<const uint32_t*>(coef + 64)[lane] - (uint32_t)v0 < 64u);  // of row `lane` of the stage
#pragma unroll 1
      for (int b = 0; b < 2; ++b) {
        f32x16 z[2];
        u32x4 p[2][2];
#pragma unroll
        for (int e = 0; e < 16; ++e) z[0][e] = z[1][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; ++kk) {
          const u32x4 a = S::fragment(from, at.rows, b, kk);
#pragma unroll
          for (int j = 0; j < 2; ++j) z[j] = mma<T>(a, wf[j][kk], z[j]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float l[4], c[4];
          load_elements<COOP_F32, 4>(lse2 + b * 32 + row_of(4 * q) + own, l);
          load_elements<COOP_F32, 4>(coef + b * 32 + row_of(4 * q) + own, c);
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int j = 0; j < 2; ++j) z[j][4 * q + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(z[j][4 * q + e], scale2, -l[e])) * c[e];
        }
        // rows whose target is among the wave's: the 1 (of coef) goes off where the target's column and the row meet
        if ((uint32_t)(hits >> (b * 32)) != 0) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            asm volatile("" ::: "memory");  // (no registers for all of the terms at once)
            const float* at_coef = coef + b * 32 + row_of(4 * q) + own;
            const u32x4 t = *reinterpret_cast<const u32x4*>(at_coef + 64);
            float c[4];
            load_elements<COOP_F32, 4>(at_coef, c);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t at_column = t[e] - (uint32_t)v0 - (uint32_t)(lane & 31);
#pragma unroll
              for (int j = 0; j < 2; ++j) z[j][4 * q + e] -= at_column == (uint32_t)(j * 32) ? c[e] : 0.f;
            }
          }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) pack<T>(z[j], p[j]);
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
          for (int c = 0; c < KS / 2; ++c) {
            const u32x4 a = S::transposed(from, at.across, b, c, s);
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[c][j] = mma<T>(a, p[j][s], acc[c][j]);
          }
      }
    });
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  const int lane = lane_anew(), own = (lane >> 5) * 4;
  if (sums != nullptr) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t v = v0 + j * 32 + (lane & 31);
      if (v >= vocab) continue;
#pragma unroll
      for (int c = 0; c < KS / 2; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int col = c * 32 + row_of(4 * q) + own;
          const float f[4] = {acc[c][j][4 * q], acc[c][j][4 * q + 1], acc[c][j][4 * q + 2], acc[c][j][4 * q + 3]};
          if (col < width) put4<COOP_F32>((char*)(sums + ((int64_t)split * rows + v) * width + col), f);
        }
    }
    return;
  }
  // rounded, and through LDS into whole rows: a short loop with one test for a row's end, in the place of as many as a lane has packs
  __syncthreads();
  const float u = *unlift;
  constexpr int kRow = KS * 32 + 8;  // bytes (and 8 more: the lanes' rows begin in different banks)
  static_assert(4 * 64 * kRow <= Stream::kLds, "the waves' rows lie where the stages were");
  char* mine = lds + uniform_wave_in_block() * (64 * kRow);
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int c = 0; c < KS / 2; ++c)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float f[4] = {acc[c][j][4 * q] * u, acc[c][j][4 * q + 1] * u, acc[c][j][4 * q + 2] * u, acc[c][j][4 * q + 3] * u};
        Pack<T, 4> x;
        x.set(f);
        *reinterpret_cast<u32x2*>(mine + (j * 32 + (lane & 31)) * kRow + (c * 32 + row_of(4 * q) + own) * 2) = __builtin_bit_cast(u32x2, x);
      }
  __syncthreads();
  constexpr int kPacks = KS * 4, kEach = kWave / kPacks;  // of 4 columns in a row, rows at a time
#pragma unroll 2
  for (int r = lane / kPacks; r < 64; r += kEach) {
    const int col = lane % kPacks * 4;
    const int64_t v = v0 + r;
    if (v >= vocab || col >= dim) continue;
    const Pack<T, 4> x = __builtin_bit_cast(Pack<T, 4>, *reinterpret_cast<const u32x2*>(mine + r * kRow + col * 2));
    typename Element<T>::M* to = (typename Element<T>::M*)out + v * dim + col;
    if (col + 4 <= dim) {
      x.store(to);
    } else {
#pragma unroll
      for (int e = 0; e < 3; ++e)
        if (col + e < dim) to[e] = x.x[e];
    }
  }
}

// Rows of `dim` elements into `rows` rows of `width`, zeros behind a row's end, behind the last of n rows, and in rows whose target is
// negative (null: all have one).  The hidden states and the weight in one launch: of few rows a launch is all that it costs.
struct PadJob {
  const char* in;
  const int32_t* target;
  char* out;
  int64_t n, rows;
  uint32_t blocks;  // 0: nothing to do
};
template <int T>
__global__ __launch_bounds__(kBlock) void k_xent_pad(PadJob first, PadJob second, int32_t dim, int32_t width) {
  const bool one = blockIdx.x < first.blocks;
  const PadJob& job = one ? first : second;
  const int64_t step = (int64_t)job.blocks * kBlock;
  typedef typename Element<T>::M M;
  constexpr int E = 16 / (int)sizeof(M);  // (a row of the copy is a multiple of 16 bytes)
  const int32_t packs = width / E;
  for (int64_t i = (int64_t)(blockIdx.x - (one ? 0 : first.blocks)) * kBlock + threadIdx.x; i < job.rows * packs; i += step) {
    const int64_t row = i / packs;
    const int32_t c = (int32_t)(i - row * packs) * E;
    const bool there = row < job.n && (job.target == nullptr || job.target[row] >= 0);
    const M* from = (const M*)job.in + row * dim + c;
    Pack<T, E> x;
    if (there && c + E <= dim) {
      x = Pack<T, E>::load(from);
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x.x[e] = there && c + e < dim ? from[e] : (M)0.f;
    }
    x.store((M*)job.out + row * width + c);
  }
}

// ---- the workspace ---------------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = (int64_t)512 << 20;  // of G
constexpr int64_t kMaxVocab = 0x7FFFF000;            // (a tile's row numbers stay below 2^31)

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// How a call is cut, and what of the workspace it uses for what.
//   few:    up to 32 rows.  W is read once and that is all there is to it: tiles of 32 rows of H, as many blocks as there are tiles of W.
//   narrow: rows of up to 128 elements of 16 bits, forward up to 256 where there are more than 32 of them (above).
//   else products in tiles, a piece of the vocabulary at a time.  Of 256 x 256, what a wave's registers hold, where there are enough of
//   them for the chip: the matrix units then take all that LDS gives.  Else, and in fp32, where they are sixteen times slower, of
//   128 x 128, two blocks on a CU (2,236 rows, 170 vertices, 768 elements of bf16: 148 -> 82 us).
//   Of few rows' tiles of W there are twice as many, half as large, where they would not fill the chip (16,048 vertices, 1,024 elements of
//   fp32: 43 -> 28 us).  dW is split over the rows where it has few tiles (14,644 rows, 6,570 vertices, 1 element of fp32: 885 -> 194 us).
struct XentPlan {
  int64_t n, vocab, width, ld;  // width: elements of a padded row
  int64_t rows, piece, vocab_rows, dw_rows;
  int64_t g_ld;  // bytes from row to row of G: not a power of two, or a tile's rows would all lie in the same few channels of memory
  int splits, dh_splits, dw_splits, tile;
  bool few, narrow, pad, lift;  // lift: G is in memory, in fp16
  size_t h, w, part, coef, lse2, target, undo, unlift, tops, g, sums, dw_sums, bytes;
  static int at_most(int64_t x, int64_t most) { return (int)(x < 1 ? 1 : x < most ? x : most); }
  XentPlan(int64_t n_, int64_t vocab_, int32_t dim, int dtype, bool aligned, bool grad) : n(n_), vocab(vocab_) {
    const int es = element_bytes(dtype);
    width = round_up(dim, 16 / es);
    ld = width * es;
    pad = !aligned || width != dim;
    narrow = es == 2 && width <= (grad ? 128 : 256) && (grad || n > 32);
    few = n <= 32 && !narrow;
    lift = grad && dtype == COOP_F16 && !narrow;
    tile = narrow || (es == 2 || few) && ((n + 255) / 256) * ((vocab + 255) / 256) >= 256 ? 256 : 128;
    rows = few ? 32 : round_up(n, tile);
    const int blocks = 256 * (narrow || few || tile == 128 ? 2 : 1);
    const int64_t row_tiles = few ? 1 : rows / tile, vocab_tiles = (vocab + tile - 1) / tile;
    vocab_rows = vocab_tiles * tile;
    // blocks: two of a narrow kernel or of few rows on a CU, one of the others; a multiple of 8 splits where that leaves out at most
    // an eighth of them, so that the blocks of an XCD have the same splits' tiles of W
    if (few) splits = at_most((vocab_tiles + (vocab_tiles + 511) / 512 - 1) / ((vocab_tiles + 511) / 512), 512);  // (of as many tiles each)
    else splits = at_most(blocks / row_tiles, narrow ? (vocab + 63) / 64 : vocab_tiles);
    if (!few && splits / 8 * 8 * 8 >= splits * 7) splits = splits / 8 * 8;
    piece = kPieceBytes / (rows * es) / tile * tile;
    if (piece < tile) piece = tile;
    if (piece > vocab_rows) piece = vocab_rows;
    const int64_t dh_tiles = row_tiles * ((width + tile - 1) / tile), first = piece < vocab ? piece : vocab;
    dh_splits = narrow ? splits : at_most(blocks / dh_tiles, (first * es + 4 * kWide - 1) / (4 * kWide));
    const int dw_tile = few ? 128 : tile;
    const int64_t dw_tiles = (first + dw_tile - 1) / dw_tile * ((width + dw_tile - 1) / dw_tile);
    dw_rows = narrow ? vocab_rows : round_up(first, dw_tile);
    dw_splits = narrow ? at_most(512 / vocab_tiles, (n + 63) / 64) : at_most((dw_tile == 128 ? 512 : 256) / dw_tiles, (n * es + 8 * kNarrow - 1) / (8 * kNarrow));
    size_t at = 0;
    auto take = [&](size_t b) { const size_t o = at; at += (b + 255) & ~(size_t)255; return o; };
    h = take(grad ? (size_t)rows * ld : pad ? (size_t)n * ld : 0);
    w = take(pad ? (size_t)vocab * ld : 0);
    part = take(grad ? 0 : (size_t)splits * n * sizeof(RowStat));
    coef = take(grad ? (size_t)rows * 4 : 0);
    lse2 = take(grad ? (size_t)rows * 4 : 0);
    target = take(grad ? (size_t)rows * 4 : 0);
    undo = take(lift ? (size_t)rows * 4 : 0);
    unlift = take(grad ? sizeof(float) : 0);
    tops = take(grad ? 256 * sizeof(float) : 0);
    g_ld = piece * es + 256;
    g = take(grad && !narrow ? (size_t)rows * g_ld : 0);
    sums = take(grad ? (size_t)dh_splits * rows * width * 4 : 0);
    dw_sums = take(grad && dw_splits > 1 ? (size_t)dw_splits * dw_rows * width * 4 : 0);
    bytes = at + 256;
  }
};

PadJob pad_job(const void* in, int64_t n, const int32_t* target, int64_t rows, const XentPlan& p, void* out) {
  const int64_t blocks = (rows * p.ld / 16 + kBlock - 1) / kBlock;
  return PadJob{(const char*)in, target, (char*)out, n, rows, (uint32_t)(blocks < 8192 ? blocks : 8192)};
}
template <int T>
void pad(const PadJob& first, const PadJob& second, int32_t dim, const XentPlan& p, hipStream_t s) {
  COOP_LAUNCH(K_XENT_PAD, k_xent_pad<T>, dim3(first.blocks + second.blocks), dim3(kBlock), 0, s, first, second, dim, (int32_t)p.width);
}

// (blocks of more than 64 KB of LDS have to be allowed, once for each kernel and device; it costs a fraction of a microsecond)
template <typename K>
bool allow_lds(K kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) == hipSuccess;
}

bool xent_aligned(const void* hidden, const void* weight) { return (((uintptr_t)hidden | (uintptr_t)weight) & 15) == 0; }

int xent_check(const void* hidden, int64_t n, const void* weight, int64_t vocab, int32_t dim, int dtype, const int32_t* targets) {
  if (!known_dtype(dtype)) return COOP_E_ARG;
  if (n < 0 || n >= ((int64_t)1 << 24) || vocab < 1 || vocab > kMaxVocab || dim < 1 || dim > (1 << 18)) return COOP_E_ARG;
  if (n > 0 && (!hidden || !weight || !targets)) return COOP_E_NULL;
  if (!aligned_for(hidden, dtype) || !aligned_for(weight, dtype)) return COOP_E_ARG;
  return COOP_OK;
}

// what logits are multiplied by for their exponentials in base 2.  (Of a scale of 0 the least number: what lies behind the vocabulary's end
// counts as minus infinity, which times 0 would be no number.)
float scale_of(float alpha) { return alpha == 0.f ? 0x1p-126f : alpha * kLog2e; }

template <int T, int WA, int WB, int TA, int TB>
bool launch_stats(const XentPlan& p, Operand w, Operand h, float alpha, const int32_t* targets, RowStat* part, hipStream_t s) {
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> P;
  constexpr int lds = P::kLds > WA * P::kRowsB * (int)sizeof(RowStat) ? P::kLds : WA * P::kRowsB * (int)sizeof(RowStat);
  const auto kernel = k_xent_stats<T, WA, WB, TA, TB>;
  if (!allow_lds(kernel, lds)) return false;
  const int64_t row_tiles = (p.n + P::kRowsB - 1) / P::kRowsB;
  COOP_LAUNCH(K_XENT_STATS, kernel, dim3((unsigned)(row_tiles * p.splits)), dim3(P::kThreads), lds, s, w, h, p.n, p.vocab, p.width, scale_of(alpha),
              targets, p.splits, part);
  return true;
}

// f(KS), for the steps of 16 elements that a row of up to MOST steps is padded to
template <int MOST, typename F>
void with_steps(int64_t width, F&& f) {
  if (width <= 32) f(std::integral_constant<int, 2>());
  else if (width <= 64) f(std::integral_constant<int, 4>());
  else if (width <= 128) f(std::integral_constant<int, 8>());
  else if constexpr (MOST > 8) f(std::integral_constant<int, MOST>());
}

template <int T>
int forward(const XentPlan& p, const void* hidden, const void* weight, int32_t dim, const int32_t* targets, float alpha, int32_t ignore,
            float* loss, float* lse, char* ws, int32_t* bad, hipStream_t s) {
  if (p.pad) {
    pad<T>(pad_job(hidden, p.n, nullptr, p.n, p, ws + p.h), pad_job(weight, p.vocab, nullptr, p.vocab, p, ws + p.w), dim, p, s);
    hidden = ws + p.h;
    weight = ws + p.w;
  }
  const Operand w{(const char*)weight, p.ld, p.vocab, p.ld}, h{(const char*)hidden, p.ld, p.n, p.ld};
  RowStat* part = (RowStat*)(ws + p.part);
  bool ok = true;
  if (p.few) {
    ok = p.tile == 128 ? launch_stats<T, 4, 1, 1, 1>(p, w, h, alpha, targets, part, s) : launch_stats<T, 4, 1, 2, 1>(p, w, h, alpha, targets, part, s);
  } else if (!p.narrow && p.tile == 128) {
    ok = launch_stats<T, 2, 2, 2, 2>(p, w, h, alpha, targets, part, s);
  } else if (!p.narrow) {
    if constexpr (T != COOP_F32) ok = launch_stats<T, 2, 2, 4, 4>(p, w, h, alpha, targets, part, s);
  } else if constexpr (T != COOP_F32) {
    with_steps<16>(p.width, [&](auto ks) {
      constexpr int KS = decltype(ks)::value, lds = RowStream<T, KS, false, false>::kLds;
      const auto kernel = k_xent_stats_narrow<T, KS>;
      ok = allow_lds(kernel, lds);
      if (!ok) return;
      COOP_LAUNCH(K_XENT_STATS, kernel, dim3((unsigned)(p.rows / p.tile * p.splits)), dim3(256), lds, s, w, h, p.n, p.vocab, scale_of(alpha), targets,
                  p.splits, part);
    });
  }
  if (!ok) return COOP_E_HIP;
  int lanes_log2 = 0;
  while (lanes_log2 < 6 && 1 << lanes_log2 < p.splits) ++lanes_log2;
  COOP_LAUNCH(K_XENT_LOSS, k_xent_loss, dim3((unsigned)(((p.n << lanes_log2) + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, (const RowStat*)part, p.splits,
              lanes_log2, p.n, p.vocab, targets, ignore, loss, lse, bad);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

template <int T>
void write_out(const float* sums, int splits, int64_t rows, const XentPlan& p, int64_t n, int32_t dim, const float* unlift, const float* undo, void* out,
               hipStream_t s) {
  const int share = splits >= kOutWaves ? kOutWaves : 1, each = kOutWaves / share * kWave;
  const int64_t blocks = (n * ((dim + 3) / 4) + each - 1) / each;
  COOP_LAUNCH(K_XENT_OUT, k_xent_out<T>, dim3((unsigned)(blocks < 16384 ? blocks : 16384)), dim3(kOutWaves * kWave), 0, s, sums, splits, share, rows, (int32_t)p.width, n, dim,
              unlift, undo, (char*)out);
}

template <int T>
bool backward_narrow(const XentPlan& p, const Operand& w, const Operand& h, int32_t dim, float alpha, const RowTerms& term, const float* unlift,
                     void* dhidden, void* dweight, float* sums, float* dw_sums, hipStream_t s) {
  bool ok = true;
  with_steps<8>(p.width, [&](auto ks) {
    constexpr int KS = decltype(ks)::value, lds_h = RowStream<T, KS, false, true>::kLds, lds_w = RowStream<T, KS, true, true>::kLds;
    const auto kh = k_xent_dh_narrow<T, KS>;
    const auto kw = k_xent_dw_narrow<T, KS>;
    ok = allow_lds(kh, lds_h) && allow_lds(kw, lds_w);
    if (!ok) return;
    if (dhidden != nullptr) {
      COOP_LAUNCH(K_XENT_DH, kh, dim3((unsigned)(p.rows / p.tile * p.dh_splits)), dim3(256), lds_h, s, w, h, p.rows, p.vocab, alpha * kLog2e, term,
                  p.dh_splits, sums, (int32_t)p.width);
      write_out<T>(sums, p.dh_splits, p.rows, p, p.n, dim, unlift, nullptr, dhidden, s);
    }
    if (dweight != nullptr) {
      float* parts = p.dw_splits > 1 ? dw_sums : nullptr;
      COOP_LAUNCH(K_XENT_DW, kw, dim3((unsigned)(p.vocab_rows / p.tile * p.dw_splits)), dim3(256), lds_w, s, w, h, p.vocab, alpha * kLog2e, term, p.dw_splits,
                  unlift, dim, (char*)dweight, parts, p.dw_rows, (int32_t)p.width);
      if (parts != nullptr) write_out<T>(parts, p.dw_splits, p.dw_rows, p, p.vocab, dim, unlift, nullptr, dweight, s);
    }
  });
  return ok;
}

// tiles of W's (or G's) rows or columns by H's rows: WA x WB waves of TA x TB; the weight's gradient in square ones
template <int T, int WA, int WB, int TA, int TB>
bool backward_pieces(const XentPlan& p, const Operand& w, const Operand& h, int32_t dim, float alpha, const RowTerms& term, const float* unlift,
                     void* dhidden, void* dweight, char* g, float* sums, float* dw_sums, hipStream_t s) {
  constexpr int N = TA == 4 ? 4 : 2;
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> G;
  typedef Product<T, WA, WB, TA, TB, true, false, kWide> H;
  typedef Product<T, 2, 2, N, N, true, true, kNarrow> W;
  const auto kg = k_xent_g<T, WA, WB, TA, TB>;
  const auto kh = k_xent_dh<T, WA, WB, TA, TB>;
  const auto kw = k_xent_dw<T, 2, 2, N, N>;
  if (!allow_lds(kg, G::kLds) || !allow_lds(kh, H::kLds) || !allow_lds(kw, W::kLds)) return false;
  const auto tiles_of = [](int64_t n, int rows) { return (uint32_t)((n + rows - 1) / rows); };
  const uint32_t row_tiles = tiles_of(p.n, G::kRowsB), col_tiles = tiles_of(p.width, H::kRowsA), w_tiles = tiles_of(p.width, W::kRowsA);
  for (int64_t v = 0; v < p.vocab; v += p.piece) {
    const int64_t len = p.vocab - v < p.piece ? p.vocab - v : p.piece;
    const uint32_t tiles = tiles_of(len, G::kRowsA);
    COOP_LAUNCH(K_XENT_G, kg, dim3(tiles * row_tiles), dim3(G::kThreads), G::kLds, s, w, h, p.vocab, p.width, alpha * kLog2e, v, tiles, term, g, p.g_ld);
    const int64_t g_bytes = (int64_t)tiles * G::kRowsA * kElem<T>;
    if (dhidden != nullptr) {
      const Operand wt{w.base + v * p.ld, p.ld, p.ld, len}, gi{g, p.g_ld, p.rows, g_bytes};
      // (every split has something to do: the last piece may be too short for all of them, and then adds nothing to the others' sums)
      const int64_t stages = (len + H::kK - 1) / H::kK;
      const int splits = (int)(p.dh_splits < stages ? p.dh_splits : stages);
      COOP_LAUNCH(K_XENT_DH, kh, dim3(row_tiles * col_tiles * splits), dim3(H::kThreads), H::kLds, s, wt, gi, len, splits, col_tiles, row_tiles,
                  v != 0, sums, p.width);
    }
    if (dweight != nullptr) {
      if (term.undo != nullptr) {
        const int64_t groups = (p.n + kWave - 1) / kWave, most = (g_bytes + kBlock * 16 - 1) / (kBlock * 16);  // (some 1,024 blocks)
        COOP_LAUNCH(K_XENT_LOWER, k_xent_lower, dim3((unsigned)groups, (unsigned)XentPlan::at_most(1024 / groups, most)), dim3(kBlock), 0, s,
                    (const float*)term.undo, p.n, g_bytes, p.g_ld, g);
      }
      const Operand ht{h.base, p.ld, p.ld, p.n}, gt{g, p.g_ld, g_bytes, p.rows};
      float* parts = p.dw_splits > 1 ? dw_sums : nullptr;
      COOP_LAUNCH(K_XENT_DW, kw, dim3(tiles_of(len, W::kRowsB) * w_tiles * p.dw_splits), dim3(W::kThreads), W::kLds, s, ht, gt, p.n, p.dw_splits, p.vocab,
                  v, dim, w_tiles, unlift, (char*)dweight, parts, p.dw_rows, p.width);
      if (parts != nullptr) write_out<T>(parts, p.dw_splits, p.dw_rows, p, len, dim, unlift, nullptr, (char*)dweight + v * dim * kElem<T>, s);
    }
  }
  return true;
}

template <int T>
int backward(const XentPlan& p, const void* hidden, const void* weight, int32_t dim, const int32_t* targets, float alpha, int32_t ignore,
             const float* lse, const float* dloss, void* dhidden, void* dweight, char* ws, int32_t* bad, hipStream_t s) {
  const RowTerms term{(float*)(ws + p.coef), (float*)(ws + p.lse2), (int32_t*)(ws + p.target), p.lift ? (float*)(ws + p.undo) : nullptr};
  float* unlift = (float*)(ws + p.unlift);
  float *sums = (float*)(ws + p.sums), *dw_sums = (float*)(ws + p.dw_sums);
  float* tops = (float*)(ws + p.tops);
  const int n_tops = T == COOP_F32 || p.n <= kTopRows ? 0 : 256;
  if (n_tops != 0) COOP_LAUNCH(K_XENT_TERMS, k_xent_top, dim3(n_tops), dim3(1024), 0, s, targets, ignore, dloss, alpha, p.n, p.vocab, tops);
  COOP_LAUNCH(K_XENT_TERMS, (k_xent_terms<T != COOP_F32>), dim3((unsigned)((p.rows + 1023) / 1024)), dim3(1024), 0, s, targets, ignore, lse, dloss,
              alpha, kOne<T>, p.n, p.rows, p.vocab, tops, n_tops, term, unlift, bad);
  pad<T>(pad_job(hidden, p.n, term.target, p.rows, p, ws + p.h), p.pad ? pad_job(weight, p.vocab, nullptr, p.vocab, p, ws + p.w) : PadJob{}, dim, p, s);
  if (p.pad) weight = ws + p.w;
  hidden = ws + p.h;
  const Operand w{(const char*)weight, p.ld, p.vocab, p.ld}, h{(const char*)hidden, p.ld, p.n, p.ld};
  if constexpr (T != COOP_F32)
    if (p.narrow) {
      if (!backward_narrow<T>(p, w, h, dim, alpha, term, unlift, dhidden, dweight, sums, dw_sums, s)) return COOP_E_HIP;
      return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
    }
  bool ok = true;
  const auto pieces = [&](auto wa, auto wb, auto ta, auto tb) {
    ok = backward_pieces<T, decltype(wa)::value, decltype(wb)::value, decltype(ta)::value, decltype(tb)::value>(p, w, h, dim, alpha, term, unlift, dhidden,
                                                                                                       dweight, ws + p.g, sums, dw_sums, s);
  };
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  typedef std::integral_constant<int, 4> Four;
  if (p.few && p.tile == 128) pieces(Four(), One(), One(), One());
  else if (p.few) pieces(Four(), One(), Two(), One());
  else if (p.tile == 128) pieces(Two(), Two(), Two(), Two());
  else if constexpr (T != COOP_F32) pieces(Two(), Two(), Four(), Four());
  if (!ok) return COOP_E_HIP;
  if (dhidden != nullptr) write_out<T>(sums, p.dh_splits, p.rows, p, p.n, dim, unlift, term.undo, dhidden, s);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" size_t coop_softmax_xent_workspace_bytes(int64_t n, int64_t vocab, int32_t dim, int dtype, int aligned, int grad) {
  if (xent_check(nullptr, 0, nullptr, vocab, dim, dtype, nullptr) != COOP_OK || n < 0 || n >= ((int64_t)1 << 24)) return 0;
  return n == 0 ? 256 : XentPlan(n, vocab, dim, dtype, aligned != 0, grad != 0).bytes;
}

extern "C" int coop_softmax_xent(const void* hidden, int64_t n, const void* weight, int64_t vocab, int32_t dim, int dtype,
                                 const int32_t* targets, float alpha, int32_t ignore, float* loss_out, float* lse_out, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  const int rc = xent_check(hidden, n, weight, vocab, dim, dtype, targets);
  if (rc != COOP_OK) return rc;
  if (n == 0) return COOP_OK;
  if (!loss_out || !lse_out || !workspace) return COOP_E_NULL;
  const XentPlan p(n, vocab, dim, dtype, xent_aligned(hidden, weight), false);
  if (workspace_bytes < p.bytes || ((uintptr_t)workspace & 255) != 0) return COOP_E_ARG;
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  int r = COOP_OK;
  with_dtype(dtype, [&](auto t) {
    r = forward<decltype(t)::value>(p, hidden, weight, dim, targets, alpha, ignore, loss_out, lse_out, (char*)workspace, bad, (hipStream_t)stream);
  });
  return r;
}

extern "C" int coop_softmax_xent_grad(const void* hidden, int64_t n, const void* weight, int64_t vocab, int32_t dim, int dtype,
                                      const int32_t* targets, float alpha, int32_t ignore, const float* lse, const float* dloss, void* dhidden,
                                      void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = xent_check(hidden, n, weight, vocab, dim, dtype, targets);
  if (rc != COOP_OK) return rc;
  if (!aligned_for(dhidden, dtype) || !aligned_for(dweight, dtype)) return COOP_E_ARG;
  if (!dhidden && !dweight) return COOP_OK;
  if (n == 0) {
    if (dweight != nullptr) clear_bytes(dweight, vocab * dim * element_bytes(dtype), (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
  }
  if (!lse || !dloss || !workspace) return COOP_E_NULL;
  const XentPlan p(n, vocab, dim, dtype, xent_aligned(hidden, weight), true);
  if (workspace_bytes < p.bytes || ((uintptr_t)workspace & 255) != 0) return COOP_E_ARG;
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  int r = COOP_OK;
  with_dtype(dtype, [&](auto t) {
    r = backward<decltype(t)::value>(p, hidden, weight, dim, targets, alpha, ignore, lse, dloss, dhidden, dweight, (char*)workspace, bad,
                                     (hipStream_t)stream);
  });
  return r;
}
