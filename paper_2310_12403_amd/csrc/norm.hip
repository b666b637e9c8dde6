// Layer norm over the last dimension: y = (x - mean) rstd w + b with rstd = 1 / sqrt(var + eps), and its gradient: with
// h = (x - mean) rstd and d = w dy,  dx = rstd (d - mean(d) - h mean(d h)),  dw = sum over rows of dy h,  db = sum over rows of dy.
//
// Bound by HBM: a row stays in the registers of the lanes that share it between its sums and its result, so that x is read once and
// y written once (backward: x and dy once, dx once).  The variance is the mean square of x - mean, taken in registers when the mean
// is there.  The weight's gradient: every lane adds up its own columns over the rows that its group takes, a block adds up its
// groups' through LDS and leaves one row of partial sums, and a second kernel adds those up.  No atomics: the same input gives the
// same bits.  The next row is asked for while one is worked on.
// 572,596 rows of 128 elements of bf16: forward 63 us, 4.7 TB/s; backward 81 us, 5.4 TB/s, and 6 to add up its blocks' sums.
#include <type_traits>

#include "coop_internal.h"
#include "elements.h"

namespace coop {
namespace {

struct NormShape {
  int64_t rows;
  int32_t dim;
  int lanes, lanes_log2;  // lanes that share a row, when a row has no more than a wave
  float eps;
};

// Where a lane's columns are.  A row is cut into packs of E columns, dealt to the lanes in order, K per lane; the last pack is anchored
// at the row's end, and the columns that it shares with the one in front do not count (`own` is the first that does).
template <int E>
struct Columns {
  int32_t at;
  int own;
  bool live;
  __device__ __forceinline__ Columns(int32_t pack, int32_t dim) {
    const int32_t c = pack * E, last = dim - E;
    live = c < dim;
    at = !live ? 0 : c < last ? c : last;
    own = live ? c - at : E;
  }
};

// Sum over the lanes that share a row: WAVES = 1: an aligned group of them in a wave; else the whole block.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, int lanes, float* lds /* [WAVES] */) {
  if constexpr (WAVES == 1) {
    return group_sum(v, lanes);
  } else {
    v = group_sum(v, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[wave_in_block()] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += lds[w];
    return t;
  }
}
template <int WAVES>
__device__ __forceinline__ void row_sums(float& a, float& b, int lanes, float* lds /* [2 WAVES] */) {
  if constexpr (WAVES == 1) {
    a = group_sum(a, lanes);
    b = group_sum(b, lanes);
  } else {
    a = group_sum(a, kWave);
    b = group_sum(b, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[2 * wave_in_block()] = a, lds[2 * wave_in_block() + 1] = b;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) a += lds[2 * w], b += lds[2 * w + 1];
  }
}

template <int WAVES> constexpr int kNormBlock = WAVES == 1 ? kBlock : WAVES * kWave;

// which rows a block takes: its first group's row, rows from group to group of the grid, and this lane's group in the block
template <int WAVES>
struct Rows {
  int64_t first, step;
  int lane, group;
  __device__ __forceinline__ explicit Rows(const NormShape& sh) {
    if constexpr (WAVES == 1) {
      const int per_block = kBlock >> sh.lanes_log2;
      group = threadIdx.x >> sh.lanes_log2;
      lane = threadIdx.x & (sh.lanes - 1);
      first = (int64_t)blockIdx.x * per_block + group;
      step = (int64_t)gridDim.x * per_block;
    } else {
      group = 0;
      lane = threadIdx.x;
      first = blockIdx.x;
      step = gridDim.x;
    }
  }
  __device__ __forceinline__ int lanes(const NormShape& sh) const { return WAVES == 1 ? sh.lanes : WAVES * kWave; }
};

// a lane's K packs of a row, as they are in memory
template <int T, int E, int K>
struct RowPacks {
  Pack<T, E> x[K];
  __device__ __forceinline__ void load(const char* row, int lane, int lanes, int32_t dim) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(lane + k * lanes, dim);
      x[k] = Pack<T, E>::load_nt(row + (int64_t)c.at * (int64_t)sizeof(typename Element<T>::M));  // (a lane without columns: the first ones)
    }
  }
};

// A lane's columns of the weight or the bias: kept in registers over all rows, or read anew for each.  Kept with two packs a lane, whose
// reads would wait for each other (445,906 rows of 602 elements of bf16 372 -> 281 us forward, 444 -> 374 backward; 32,768 of 8,192 of fp32
// forward 410 -> 365), but not beside the sums of rows on sixteen waves (16,384 of 16,384 of bf16 backward 456 -> 587); of one pack they are
// as soon read (2,097,152 rows of 128 of fp32 forward 420, kept 450).
template <int W, int E, int K, bool kKept>
struct LaneWeights {
  float x[kKept ? K : 1][E];
  const char* p;
  __device__ __forceinline__ LaneWeights(const char* p_, int lane, int lanes, int32_t dim) : p(p_) {
    if (!kKept || p == nullptr) return;
#pragma unroll
    for (int k = 0; k < (kKept ? K : 0); ++k) load_elements<W, E>(p + (int64_t)Columns<E>(lane + k * lanes, dim).at * (int64_t)sizeof(typename Element<W>::M), x[k]);
  }
  __device__ __forceinline__ void get(int k, int32_t at, float (&f)[E]) const {  // (only where there are any)
    if constexpr (kKept) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = x[k][e];
    } else {
      load_elements<W, E>(p + (int64_t)at * (int64_t)sizeof(typename Element<W>::M), f);
    }
  }
};

// (y may be x: neither is told to be apart from the other.  A row is read whole before any of it is written.)
template <int T, int W, int E, int K, int WAVES>
__global__ __launch_bounds__(kNormBlock<WAVES>) void k_norm(const char* x, NormShape sh, const char* __restrict__ weight,
                                                            const char* __restrict__ bias, char* y, float* __restrict__ mean_out,
                                                            float* __restrict__ rstd_out) {
  __shared__ float lds[WAVES];
  const Rows<WAVES> rows(sh);
  const int lanes = rows.lanes(sh);
  const int64_t row_bytes = (int64_t)sh.dim * (int64_t)sizeof(typename Element<T>::M);
  const float n = (float)sh.dim;
  const LaneWeights<W, E, K, K == 2> w_of(weight, rows.lane, lanes, sh.dim), b_of(bias, rows.lane, lanes, sh.dim);
  RowPacks<T, E, K> next;  // (the next row is on its way while this one is worked on)
  if (rows.first < sh.rows) next.load(x + rows.first * row_bytes, rows.lane, lanes, sh.dim);
  for (int64_t r = rows.first; r < sh.rows; r += rows.step) {
    float f[K][E];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) next.x[k].get(f[k]);
    if (r + rows.step < sh.rows) next.load(x + (r + rows.step) * row_bytes, rows.lane, lanes, sh.dim);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += e >= c.own ? f[k][e] : 0.f;
    }
    const float mean = row_sum<WAVES>(sum, lanes, lds) / n;
    float square = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        f[k][e] -= mean;
        square += e >= c.own ? f[k][e] * f[k][e] : 0.f;
      }
    }
    const float rstd = 1.f / sqrtf(row_sum<WAVES>(square, lanes, lds) / n + sh.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      if (!c.live) continue;
      float w[E], b[E];
      if (weight != nullptr) w_of.get(k, c.at, w);
      if (bias != nullptr) b_of.get(k, c.at, b);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        float v = f[k][e] * rstd;
        if (weight != nullptr) v *= w[e];
        if (bias != nullptr) v += b[e];
        f[k][e] = v;
      }
      Pack<T, E> out;
      out.set(f[k]);
      out.store_nt(y + r * row_bytes + (int64_t)c.at * (int64_t)sizeof(typename Element<T>::M));
    }
    if (rows.lane == 0) {
      mean_out[r] = mean;
      rstd_out[r] = rstd;
    }
  }
}

// Rows on sixteen waves with 32 columns a lane or more: the sums for the weight's gradient do not fit beside them into the 128 registers of
// a lane, and are a kernel's of their own.  (16,384 rows of 16,384 elements of bf16, 16 columns: 458 us, and 500 with the second kernel.)
template <int E, int K, int WAVES> constexpr bool kSumsApart = WAVES == 16 && E * K >= 32;

// part: [gridDim.x][2][dim], the block's sums of dy h and of dy (null: not asked for, or not here).  (dx may be dy, as y may be x above.)
template <int T, int W, int E, int K, int WAVES>
__global__ __launch_bounds__(kNormBlock<WAVES>) void k_norm_grad(const char* dy, const char* __restrict__ x, NormShape sh,
                                                                 const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                                                 const char* __restrict__ weight, char* dx,
                                                                 float* __restrict__ part) {
  constexpr int kLds = WAVES == 1 ? kBlock * E : 2 * WAVES;
  __shared__ float lds[kLds];
  const Rows<WAVES> rows(sh);
  const int lanes = rows.lanes(sh);
  const int64_t row_bytes = (int64_t)sh.dim * (int64_t)sizeof(typename Element<T>::M);
  const float n = (float)sh.dim;
  const LaneWeights<W, E, K, K == 2 && WAVES < 16> w_of(weight, rows.lane, lanes, sh.dim);
  float dw[K][E], db[K][E];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int e = 0; e < E; ++e) dw[k][e] = db[k][e] = 0.f;
  RowPacks<T, E, K> next_x, next_dy;  // (as in the forward kernel)
  float next_mean = 0.f, next_rstd = 0.f;
  const auto look_ahead = [&](int64_t r) {
    next_x.load(x + r * row_bytes, rows.lane, lanes, sh.dim);
    next_dy.load(dy + r * row_bytes, rows.lane, lanes, sh.dim);
    next_mean = mean_in[r];
    next_rstd = rstd_in[r];
  };
  if (rows.first < sh.rows) look_ahead(rows.first);
  for (int64_t r = rows.first; r < sh.rows; r += rows.step) {
    const float mean = next_mean, rstd = next_rstd;
    float h[K][E], d[K][E];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      next_x.x[k].get(h[k]);
      next_dy.x[k].get(d[k]);
    }
    if (r + rows.step < sh.rows) look_ahead(r + rows.step);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      float w[E];
      if (weight != nullptr) w_of.get(k, c.at, w);  // (of a lane without columns those of the first: it writes nothing, and its sums count nothing)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        h[k][e] = (h[k][e] - mean) * rstd;
        if constexpr (!kSumsApart<E, K, WAVES>) {
          dw[k][e] += d[k][e] * h[k][e];
          db[k][e] += d[k][e];
        }
        if (weight != nullptr) d[k][e] *= w[e];
        s1 += e >= c.own ? d[k][e] : 0.f;
        s2 += e >= c.own ? d[k][e] * h[k][e] : 0.f;
      }
    }
    row_sums<WAVES>(s1, s2, lanes, lds);
    s1 /= n;
    s2 /= n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      if (!c.live) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) d[k][e] = (d[k][e] - s1 - h[k][e] * s2) * rstd;
      Pack<T, E> out;
      out.set(d[k]);
      out.store_nt(dx + r * row_bytes + (int64_t)c.at * (int64_t)sizeof(typename Element<T>::M));
    }
  }
  if (kSumsApart<E, K, WAVES> || part == nullptr) return;
  float* to = part + (int64_t)blockIdx.x * 2 * sh.dim;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float* sums = q == 0 ? dw[k] : db[k];
      if constexpr (WAVES == 1) {  // the block's groups have the same columns: the first adds up all of them
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) lds[e * kBlock + threadIdx.x] = sums[e];
        __syncthreads();
        if (rows.group == 0)
          for (int g = 1; g < kBlock >> sh.lanes_log2; ++g)
#pragma unroll
            for (int e = 0; e < E; ++e) sums[e] += lds[e * kBlock + (g << sh.lanes_log2) + rows.lane];
      }
      if (rows.group == 0)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e >= c.own) to[(int64_t)q * sh.dim + c.at + e] = sums[e];
    }
  }
}

// part[split]: the sums of dy h and of dy over every splits-th four rows, of 64 E columns a block; a wave has every fourth row.  (8,192 rows of
// 32,768 elements of bf16, weight and all: 1,587 -> 686 us, x and dy read twice.)
template <int T, int E>
__global__ __launch_bounds__(kBlock) void k_norm_sums(const char* __restrict__ dy, const char* __restrict__ x, NormShape sh,
                                                      const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ part) {
  __shared__ float lds[kWavesPerBlock][2 * E][kWave];
  const Columns<E> c((int32_t)blockIdx.x * kWave + lane_id(), sh.dim);
  const int64_t row_bytes = (int64_t)sh.dim * (int64_t)sizeof(typename Element<T>::M), at = (int64_t)c.at * (int64_t)sizeof(typename Element<T>::M);
  const int wave = uniform_wave_in_block();
  float sums[2 * E];
#pragma unroll
  for (int e = 0; e < 2 * E; ++e) sums[e] = 0.f;
#pragma unroll 4
  for (int64_t r = (int64_t)blockIdx.y * kWavesPerBlock + wave; r < sh.rows; r += (int64_t)gridDim.y * kWavesPerBlock) {
    const float m = mean[r], s = rstd[r];
    float h[E], d[E];
    Pack<T, E>::load_nt(x + r * row_bytes + at).get(h);
    Pack<T, E>::load_nt(dy + r * row_bytes + at).get(d);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      sums[e] += d[e] * ((h[e] - m) * s);
      sums[E + e] += d[e];
    }
  }
#pragma unroll
  for (int e = 0; e < 2 * E; ++e) lds[wave][e][lane_id()] = sums[e];
  __syncthreads();
  if (wave != 0 || !c.live) return;
  float* to = part + (int64_t)blockIdx.y * 2 * sh.dim;
#pragma unroll
  for (int e = 0; e < 2 * E; ++e) {
    float t = sums[e];
#pragma unroll
    for (int w = 1; w < kWavesPerBlock; ++w) t += lds[w][e][lane_id()];
    if (e % E >= c.own) to[(int64_t)(e / E) * sh.dim + c.at + e % E] = t;
  }
}

// out[c] = sum over the blocks of part[b][c], c < 2 dim; a block has 64 columns, its waves deal the rows among themselves
constexpr int kJoinWaves = 16;
__global__ __launch_bounds__(kJoinWaves* kWave) void k_norm_join(const float* __restrict__ part, int blocks, int32_t dim, float* __restrict__ dw,
                                                                 float* __restrict__ db) {
  __shared__ float lds[kJoinWaves][kWave];
  const int64_t c = (int64_t)blockIdx.x * kWave + lane_id(), width = 2 * (int64_t)dim;
  float sum = 0.f;
  if (c < width) {
#pragma unroll 16
    for (int b = wave_in_block(); b < blocks; b += kJoinWaves) sum += part[b * width + c];
  }
  lds[wave_in_block()][lane_id()] = sum;
  __syncthreads();
  if (wave_in_block() != 0 || c >= width) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < kJoinWaves; ++w) sum += lds[w][lane_id()];
  if (c < dim) {
    if (dw != nullptr) dw[c] = sum;
  } else if (db != nullptr) {
    db[c - dim] = sum;
  }
}

// How a row is shared: K packs a lane on one wave or less, on 4 or on 16 waves, as few lanes as hold it.
struct NormLayout { int e, k, waves, lanes, lanes_log2; };
bool norm_layout(int32_t dim, int dtype, NormLayout* out) {
  const int e = dtype == COOP_F32 ? 4 : 8;
  NormLayout l{dim >= e ? e : 1, 1, 1, 1, 0};
  const int32_t packs = (dim + l.e - 1) / l.e;
  if (packs <= 4 * kWave) {
    while (l.lanes < packs && l.lanes < kWave) l.lanes *= 2, ++l.lanes_log2;
    while (l.k * l.lanes < packs) l.k *= 2;
  } else {
    l.waves = packs <= 4 * 4 * kWave ? 4 : 16;
    l.lanes = l.waves * kWave;
    while (l.k * l.lanes < packs) l.k *= 2;
  }
  *out = l;
  return l.k <= 8;
}

// Blocks of a pass: as many as are on the chip at once (the gradient's registers: 5, 3 or 2 blocks of four waves a CU), and for a
// gradient no more than leave each group two rows.
int64_t norm_blocks(int64_t rows, const NormLayout& l, bool grad) {
  const int64_t per_block = l.waves == 1 ? kBlock / l.lanes : 1;
  int64_t b = (rows + per_block - 1) / per_block;
  const int64_t each = l.waves == 16 ? (grad ? 1 : 2) : !grad ? 8 : l.k == 1 ? 5 : l.k == 2 ? 3 : 2, most = 256 * each;
  if (b > most) b = most;
  if (grad && b > rows / (2 * per_block) + 1) b = rows / (2 * per_block) + 1;
  return b;
}

template <int T, int W, typename F>
void with_layout(const NormLayout& l, F&& f) {
  constexpr int E = T == COOP_F32 ? 4 : 8;
  const auto k = [&](auto waves, auto wide) {
    constexpr int N = decltype(waves)::value;
    if (l.k == 1) f(std::integral_constant<int, decltype(wide)::value>(), std::integral_constant<int, 1>(), std::integral_constant<int, N>());
    if constexpr (decltype(wide)::value != 1) {
      if (l.k == 2) f(std::integral_constant<int, decltype(wide)::value>(), std::integral_constant<int, 2>(), std::integral_constant<int, N>());
      if (l.k == 4) f(std::integral_constant<int, decltype(wide)::value>(), std::integral_constant<int, 4>(), std::integral_constant<int, N>());
      if constexpr (N == 16)
        if (l.k == 8) f(std::integral_constant<int, decltype(wide)::value>(), std::integral_constant<int, 8>(), std::integral_constant<int, N>());
    }
  };
  if (l.e == 1) k(std::integral_constant<int, 1>(), std::integral_constant<int, 1>());
  else if (l.waves == 1) k(std::integral_constant<int, 1>(), std::integral_constant<int, E>());
  else if (l.waves == 4) k(std::integral_constant<int, 4>(), std::integral_constant<int, E>());
  else k(std::integral_constant<int, 16>(), std::integral_constant<int, E>());
}

template <typename F>
void with_types(int dtype, int weight_dtype, F&& f) {
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    if (weight_dtype == COOP_F32) f(std::integral_constant<int, T>(), std::integral_constant<int, COOP_F32>());
    else if constexpr (T != COOP_F32) f(std::integral_constant<int, T>(), std::integral_constant<int, T>());
  });
}

int norm_check(int64_t rows, int32_t dim, int dtype, int weight_dtype, NormLayout* l) {
  if (!known_dtype(dtype) || (weight_dtype != COOP_F32 && weight_dtype != dtype)) return COOP_E_ARG;
  if (rows < 0 || dim < 1 || !norm_layout(dim, dtype, l)) return COOP_E_ARG;
  return COOP_OK;
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" int coop_layer_norm(const void* x, int64_t n_rows, int32_t dim, int dtype, const void* weight, const void* bias, int weight_dtype,
                               float eps, void* out, float* mean_out, float* rstd_out, void* stream) {
  NormLayout l;
  const int rc = norm_check(n_rows, dim, dtype, weight_dtype, &l);
  if (rc != COOP_OK) return rc;
  if (!(eps >= 0.f)) return COOP_E_ARG;
  if (n_rows == 0) return COOP_OK;
  if (!x || !out || !mean_out || !rstd_out) return COOP_E_NULL;
  if (!aligned_for(x, dtype) || !aligned_for(out, dtype) || !aligned_for(weight, weight_dtype) || !aligned_for(bias, weight_dtype)) return COOP_E_ARG;
  const NormShape sh{n_rows, dim, l.lanes, l.lanes_log2, eps};
  const dim3 grid((unsigned)norm_blocks(n_rows, l, false));
  with_types(dtype, weight_dtype, [&](auto t, auto w) {
    constexpr int T = decltype(t)::value, W = decltype(w)::value;
    with_layout<T, W>(l, [&](auto e, auto k, auto waves) {
      constexpr int E = decltype(e)::value, K = decltype(k)::value, N = decltype(waves)::value;
      COOP_LAUNCH(K_NORM, (k_norm<T, W, E, K, N>), grid, dim3(kNormBlock<N>), 0, (hipStream_t)stream, (const char*)x, sh, (const char*)weight,
                  (const char*)bias, (char*)out, mean_out, rstd_out);
    });
  });
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_layer_norm_grad_workspace_bytes(int64_t n_rows, int32_t dim, int dtype) {
  NormLayout l;
  if (norm_check(n_rows, dim, dtype, dtype, &l) != COOP_OK) return 0;
  return (size_t)norm_blocks(n_rows, l, true) * 2 * (size_t)dim * sizeof(float) + 256;
}

extern "C" int coop_layer_norm_grad(const void* dy, const void* x, int64_t n_rows, int32_t dim, int dtype, const float* mean, const float* rstd,
                                    const void* weight, int weight_dtype, void* dx, float* dweight, float* dbias, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  NormLayout l;
  const int rc = norm_check(n_rows, dim, dtype, weight_dtype, &l);
  if (rc != COOP_OK) return rc;
  const bool sums = dweight != nullptr || dbias != nullptr;
  if (n_rows > 0 && (!dy || !x || !mean || !rstd || !dx)) return COOP_E_NULL;
  if (sums && !workspace) return COOP_E_NULL;
  if (!aligned_for(x, dtype) || !aligned_for(dy, dtype) || !aligned_for(dx, dtype) || !aligned_for(weight, weight_dtype)) return COOP_E_ARG;
  if (sums && (workspace_bytes < coop_layer_norm_grad_workspace_bytes(n_rows, dim, dtype) || ((uintptr_t)workspace & 15) != 0)) return COOP_E_ARG;
  hipStream_t s = (hipStream_t)stream;
  const NormShape sh{n_rows, dim, l.lanes, l.lanes_log2, 0.f};
  int64_t blocks = norm_blocks(n_rows, l, true);
  float* part = sums ? (float*)workspace : nullptr;
  if (n_rows > 0)
    with_types(dtype, weight_dtype, [&](auto t, auto w) {
      constexpr int T = decltype(t)::value, W = decltype(w)::value;
      with_layout<T, W>(l, [&](auto e, auto k, auto waves) {
        constexpr int E = decltype(e)::value, K = decltype(k)::value, N = decltype(waves)::value;
        const unsigned grid = (unsigned)blocks;
        if constexpr (kSumsApart<E, K, N>)
          if (sums) {  // (before dx, which may lie where dy does; no more splits than the workspace has rows for, some 2,048 blocks)
            const int64_t tiles = (dim + kWave * E - 1) / (kWave * E), splits = 2048 / tiles + 1;
            if (splits < blocks) blocks = splits;
            COOP_LAUNCH(K_NORM_GRAD, (k_norm_sums<T, E>), dim3((unsigned)tiles, (unsigned)blocks), dim3(kBlock), 0, s, (const char*)dy, (const char*)x, sh,
                        mean, rstd, part);
          }
        COOP_LAUNCH(K_NORM_GRAD, (k_norm_grad<T, W, E, K, N>), dim3(grid), dim3(kNormBlock<N>), 0, s, (const char*)dy, (const char*)x,
                    sh, mean, rstd, (const char*)weight, (char*)dx, part);
      });
    });
  if (sums)
    COOP_LAUNCH(K_NORM_JOIN, k_norm_join, dim3((unsigned)((2 * (int64_t)dim + kWave - 1) / kWave)), dim3(kJoinWaves * kWave), 0, s,
                (const float*)part, n_rows > 0 ? (int)blocks : 0, dim, dweight, dbias);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
