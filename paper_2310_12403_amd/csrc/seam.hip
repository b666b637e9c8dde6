// The seam between two blocks of a residual model: r = alpha x + gate N_after(f), y = N_before(r), and its gradient.  x is the residual stream,
// f a block's output, r the stream behind it and y the next block's input; N is a layer norm or a root-mean-square norm with its weights, either
// of the two may be missing, and so may the gate, which is one for each column or one for each element.
//
// Backward, with h = (v - mean) rstd the normed rows of either, p = N_after(f), c(d) = d - avg(d) - h avg(d h) (root mean square: without
// avg(d)) and dr the gradient that comes along the stream:
//   d = dr + rstd2 c(dy w2),  dx = alpha d,  dgate = d p,  e = d gate,  df = rstd1 c(e w1),
//   dw2 = sum dy h2, db2 = sum dy, dw1 = sum e h1, db1 = sum e.
// r is made once more from x and f by the instructions that made it: as it is stored it would have been rounded, and h2 with it.
// Where the gate is one for each column, its gradient and those of N_after's weights are sums of d h1 and of d times what the columns have,
// so that four sums are all that a lane holds for each of its columns.
//
// Bound by HBM, and laid out as the layer norm: a row stays in the registers of the lanes that share it, everything is read once and written
// once, the next row is asked for while one is worked on, and sums over the rows are a lane's, a block's and then a second kernel's.
#include <type_traits>

#include "coop_internal.h"
#include "rows.h"

namespace coop {
namespace {

struct SeamShape {
  int64_t rows;
  int32_t dim;
  int lanes, lanes_log2;  // lanes that share a row, when a row has no more than a wave
  float eps, alpha;
  bool after, before, rms;
  int gate;     // COOP_GATE_..
  bool wide_w;  // weights, biases and the columns' gate are fp32
  bool last_in_lds;  // N_before's bias is, where the others are
};

constexpr int kColumnGate = COOP_GATE_COLUMNS, kRowGate = COOP_GATE_ELEMENTS;

// a lane's K packs of E elements of a row, as they are in memory, 16 bytes at a time where they are longer
template <int T, int E, int K>
struct SeamPacks {
  static constexpr int kSize = (int)sizeof(typename Element<T>::M), kParts = E * kSize <= 16 ? 1 : E * kSize / 16, kEach = E / kParts;
  Pack<T, kEach> x[K][kParts];
  __device__ __forceinline__ void load(const char* row, int lane, int lanes, int32_t dim) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(lane + k * lanes, dim);
#pragma unroll
      for (int i = 0; i < kParts; ++i) x[k][i] = Pack<T, kEach>::load_nt(row + ((int64_t)c.at + i * kEach) * kSize);
    }
  }
  __device__ __forceinline__ void get(int k, float (&f)[E]) const {
#pragma unroll
    for (int i = 0; i < kParts; ++i)
#pragma unroll
      for (int e = 0; e < kEach; ++e) f[i * kEach + e] = (float)x[k][i].x[e];
  }
};
template <int T, int E>
__device__ __forceinline__ void put_pack(char* at, const float (&f)[E]) {
  constexpr int kSize = (int)sizeof(typename Element<T>::M), kParts = E * kSize <= 16 ? 1 : E * kSize / 16, kEach = E / kParts;
#pragma unroll
  for (int i = 0; i < kParts; ++i) {
    Pack<T, kEach> x;
#pragma unroll
    for (int e = 0; e < kEach; ++e) x.x[e] = (typename Element<T>::M)f[i * kEach + e];
    x.store_nt(at + i * kEach * kSize);
  }
}

// The vectors of weights that there are, in 32 bits one behind the other in LDS: read anew for each row, and not from memory, where a read would wait
// for all of the next row, which was asked for before it.  (Rows too wide for that read them from memory.)
struct SeamWeightPointers { const char *gate, *w1, *b1, *w2, *b2; };
constexpr int32_t kSeamLdsDim = 4096;
template <int T, int E, bool WHOLE>
struct SeamWeights {
  const char* p;
  const float* lds;  // null: from memory
  bool wide;
  float other;  // where there is no such vector
  // all threads of the block; `next` is moved behind it
  __device__ __forceinline__ SeamWeights(const char* p_, bool wide_, float other_, int32_t dim, float*& next) : p(p_), lds(nullptr), wide(wide_), other(other_) {
    if (p == nullptr || dim > kSeamLdsDim) return;
    for (int32_t i = threadIdx.x; i < dim; i += blockDim.x) next[i] = wide ? ((const float*)p)[i] : (float)((const typename Element<T>::M*)p)[i];
    lds = next;
    next += (dim + 3) & ~3;
  }
  __device__ __forceinline__ void get(int32_t at, float (&f)[E]) const {
    if (p == nullptr) {
#pragma unroll
      for (int e = 0; e < E; ++e) f[e] = other;
    } else if (lds != nullptr) {
      typedef float Four __attribute__((ext_vector_type(4)));
      if constexpr (WHOLE && E % 4 == 0) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
          const Four x = *reinterpret_cast<const Four*>(lds + at + i);
#pragma unroll
          for (int e = 0; e < 4; ++e) f[i + e] = x[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = lds[at + e];
      }
    } else if (wide) {
      load_elements<COOP_F32, E>(p + (int64_t)at * 4, f);
    } else {
      load_elements<T, E>(p + (int64_t)at * (int64_t)sizeof(typename Element<T>::M), f);
    }
  }
};
inline int seam_lds(const SeamWeightPointers& wp, bool columns, int32_t dim) {
  if (dim > kSeamLdsDim) return 0;
  const int n = (columns && wp.gate != nullptr) + (wp.w1 != nullptr) + (wp.b1 != nullptr) + (wp.w2 != nullptr) + (wp.b2 != nullptr);
  return n * ((dim + 3) & ~3) * 4;
}

// What a row's other lanes write to when its last pack overlaps the one in front, in place: it is here before the lanes meet.  (Within a wave loads
// and stores are in order.)
template <bool WHOLE, int WAVES, int E>
__device__ __forceinline__ void arrived(float (&v)[E]) {
  if constexpr (!WHOLE && WAVES > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) asm volatile("" : "+v"(v[e]));
  }
}

// mean and 1 / size of a row, and v left as v - mean (root mean square: mean 0)
template <int E, int K, int WAVES, bool WHOLE>
__device__ __forceinline__ void row_statistics(float (&v)[K][E], const Rows<WAVES>& rows, int lanes, const SeamShape& sh, RowSums<WAVES>& sums, float* mean_out,
                                               float* rstd_out) {
  const float n = (float)sh.dim;
  float mean = 0.f;
  if (!sh.rms) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) sum += WHOLE || e >= c.own ? v[k][e] : 0.f;
    }
    mean = sums(sum, lanes) / n;
  }
  float square = 0.f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v[k][e] -= mean;
      square += WHOLE || e >= c.own ? v[k][e] * v[k][e] : 0.f;
    }
  }
  *mean_out = mean;
  *rstd_out = 1.f / sqrtf(sums(square, lanes) / n + sh.eps);
}

// Waves of a SIMD that a kernel's registers are cut for, and that its grid fills.  (A gradient in 16 bits for 3, with 26 registers spilled, 572,596
// rows of 128: 320 us for 309 forward and backward; 3 blocks a CU where 2 fit: 393.)
constexpr int seam_waves(int e, int k, int waves, bool grad) { return k > 1 ? 2 : !grad ? 4 : waves == 8 || e == 8 ? 2 : 3; }

// stats: [4][rows], mean and rstd of N_after, mean and rstd of N_before.  (Outputs are not told to be apart from the inputs: a row is read whole
// before any of it is written.)
template <int T, int S, int E, int K, int WAVES, bool WHOLE>
__global__ __launch_bounds__(kNormBlock<WAVES>) __attribute__((amdgpu_waves_per_eu(seam_waves(E, K, WAVES, false)))) void k_seam(const char* x, const char* f, SeamWeightPointers wp, SeamShape sh, char* r_out, char* y,
                                                            float* __restrict__ stats) {
  __shared__ float lds[4 * WAVES];
  RowSums<WAVES> row_sums(lds);
  constexpr int64_t kT = (int64_t)sizeof(typename Element<T>::M), kS = (int64_t)sizeof(typename Element<S>::M);
  const Rows<WAVES> rows(sh);
  const int lanes = rows.lanes(sh);
  extern __shared__ __attribute__((aligned(16))) float weights[];
  float* next_weights = weights;
  typedef SeamWeights<T, E, WHOLE> Weights;
  const Weights gate_of(sh.gate == kColumnGate ? wp.gate : nullptr, sh.wide_w, 1.f, sh.dim, next_weights), w1_of(wp.w1, sh.wide_w, 1.f, sh.dim, next_weights);
  const Weights b1_of(wp.b1, sh.wide_w, 0.f, sh.dim, next_weights), w2_of(wp.w2, sh.wide_w, 1.f, sh.dim, next_weights);
  const Weights b2_of(wp.b2, sh.wide_w, 0.f, sh.last_in_lds ? sh.dim : kSeamLdsDim + 1, next_weights);
  __syncthreads();
  SeamPacks<S, E, K> next_x;  // (the next row is on its way while this one is worked on)
  SeamPacks<T, E, K> next_f, next_g;
  const auto look_ahead = [&](int64_t r) {
    next_x.load(x + r * sh.dim * kS, rows.lane, lanes, sh.dim);
    next_f.load(f + r * sh.dim * kT, rows.lane, lanes, sh.dim);
    if (sh.gate == kRowGate) next_g.load(wp.gate + r * sh.dim * kT, rows.lane, lanes, sh.dim);
  };
  if (rows.first < sh.rows) look_ahead(rows.first);
  for (int64_t r = rows.first; r < sh.rows; r += rows.step) {
    float v[K][E], p[K][E], g[K][E];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      next_x.get(k, v[k]);
      arrived<WHOLE, WAVES>(v[k]);
      next_f.get(k, p[k]);
      if (sh.gate == kRowGate) next_g.get(k, g[k]);
      else gate_of.get(c.at, g[k]);
    }
    if (r + rows.step < sh.rows) look_ahead(r + rows.step);
    float mean1 = 0.f, rstd1 = 1.f, mean2 = 0.f, rstd2 = 1.f;
    if (sh.after) {
      row_statistics<E, K, WAVES, WHOLE>(p, rows, lanes, sh, row_sums, &mean1, &rstd1);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const Columns<E> c(rows.lane + k * lanes, sh.dim);
        float w[E], b[E];
        w1_of.get(c.at, w);
        b1_of.get(c.at, b);
#pragma unroll
        for (int e = 0; e < E; ++e) p[k][e] = p[k][e] * rstd1 * w[e] + b[e];
      }
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = v[k][e] * sh.alpha + p[k][e] * g[k][e];
      if (sh.before || (!WHOLE && !c.live)) continue;
      put_pack<S, E>(r_out + (r * sh.dim + c.at) * kS, v[k]);
    }
    if (sh.before) {
      float out[K][E];
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) out[k][e] = v[k][e];
      row_statistics<E, K, WAVES, WHOLE>(out, rows, lanes, sh, row_sums, &mean2, &rstd2);
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const Columns<E> c(rows.lane + k * lanes, sh.dim);
        if (!WHOLE && !c.live) continue;
        float w[E], b[E];
        w2_of.get(c.at, w);
        b2_of.get(c.at, b);
#pragma unroll
        for (int e = 0; e < E; ++e) out[k][e] = out[k][e] * rstd2 * w[e] + b[e];
        put_pack<S, E>(r_out + (r * sh.dim + c.at) * kS, v[k]);
        put_pack<T, E>(y + (r * sh.dim + c.at) * kT, out[k]);
      }
    }
    if (rows.lane == 0) {
      stats[r] = mean1;
      stats[sh.rows + r] = rstd1;
      stats[2 * sh.rows + r] = mean2;
      stats[3 * sh.rows + r] = rstd2;
    }
  }
}

// part: [gridDim.x][4][dim]: the block's sums of d h1 and of d (of e, where the gate is an element's; h1 is f where there is no norm behind it),
// of dy h2 and of dy; null: not asked for.
template <int T, int S, int E, int K, int WAVES, bool WHOLE>
__global__ __launch_bounds__(kNormBlock<WAVES>) __attribute__((amdgpu_waves_per_eu(seam_waves(E, K, WAVES, true)))) void k_seam_grad(const char* dr, const char* dy, const char* __restrict__ x, const char* __restrict__ f,
                                                                 const float* __restrict__ stats, SeamWeightPointers wp, SeamShape sh, char* dx, char* df,
                                                                 char* dgate, float* __restrict__ part) {
  constexpr int kLds = WAVES == 1 ? kBlock * E : 4 * WAVES;
  __shared__ float lds[kLds];
  RowSums<WAVES> row_sums(lds);
  constexpr int64_t kT = (int64_t)sizeof(typename Element<T>::M), kS = (int64_t)sizeof(typename Element<S>::M);
  const Rows<WAVES> rows(sh);
  const int lanes = rows.lanes(sh);
  const float n = (float)sh.dim;
  extern __shared__ __attribute__((aligned(16))) float weights[];
  float* next_weights = weights;
  typedef SeamWeights<T, E, WHOLE> Weights;
  const Weights gate_of(sh.gate == kColumnGate ? wp.gate : nullptr, sh.wide_w, 1.f, sh.dim, next_weights), w1_of(wp.w1, sh.wide_w, 1.f, sh.dim, next_weights);
  const Weights b1_of(wp.b1, sh.wide_w, 0.f, sh.dim, next_weights), w2_of(wp.w2, sh.wide_w, 1.f, sh.dim, next_weights);
  __syncthreads();
  float sums[4][K][E];
#pragma unroll
  for (int q = 0; q < 4; ++q)
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int e = 0; e < E; ++e) sums[q][k][e] = 0.f;
  SeamPacks<S, E, K> next_dr, next_x;  // (as in the forward kernel)
  SeamPacks<T, E, K> next_dy, next_f, next_g;
  float next_stats[4];
  const auto look_ahead = [&](int64_t r) {
    if (dr != nullptr) next_dr.load(dr + r * sh.dim * kS, rows.lane, lanes, sh.dim);
    next_f.load(f + r * sh.dim * kT, rows.lane, lanes, sh.dim);
    if (sh.before) {
      next_x.load(x + r * sh.dim * kS, rows.lane, lanes, sh.dim);
      next_dy.load(dy + r * sh.dim * kT, rows.lane, lanes, sh.dim);
    }
    if (sh.gate == kRowGate) next_g.load(wp.gate + r * sh.dim * kT, rows.lane, lanes, sh.dim);
#pragma unroll
    for (int q = 0; q < 4; ++q) next_stats[q] = stats[q * sh.rows + r];
  };
  if (rows.first < sh.rows) look_ahead(rows.first);
  for (int64_t r = rows.first; r < sh.rows; r += rows.step) {
    const float mean1 = next_stats[0], rstd1 = next_stats[1], mean2 = next_stats[2], rstd2 = next_stats[3];
    float d[K][E], h1[K][E], h2[K][E], t[K][E], g[K][E];  // (t: dy w2, then e w1)
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      next_f.get(k, h1[k]);
      if (sh.before) next_x.get(k, h2[k]), next_dy.get(k, t[k]);
      if (sh.gate == kRowGate) next_g.get(k, g[k]);
      else gate_of.get(c.at, g[k]);
      if (dr != nullptr) {
        next_dr.get(k, d[k]);
        arrived<WHOLE, WAVES>(d[k]);
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) d[k][e] = 0.f;
      }
    }
    if (r + rows.step < sh.rows) look_ahead(r + rows.step);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      float w[E], b[E];
      if (sh.after) {
#pragma unroll
        for (int e = 0; e < E; ++e) h1[k][e] = (h1[k][e] - mean1) * rstd1;
      }
      if (!sh.before) continue;
      if (sh.after) {
        w1_of.get(c.at, w);
        b1_of.get(c.at, b);
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float p = sh.after ? h1[k][e] * w[e] + b[e] : h1[k][e];
        h2[k][e] = (h2[k][e] * sh.alpha + p * g[k][e] - mean2) * rstd2;
      }
      w2_of.get(c.at, w);
#pragma unroll
      for (int e = 0; e < E; ++e) {
        sums[2][k][e] += t[k][e] * h2[k][e];
        sums[3][k][e] += t[k][e];
        t[k][e] *= w[e];
        s1 += WHOLE || e >= c.own ? t[k][e] : 0.f;
        s2 += WHOLE || e >= c.own ? t[k][e] * h2[k][e] : 0.f;
      }
    }
    if (sh.before) {
      row_sums(s1, s2, lanes);
      s1 = sh.rms ? 0.f : s1 / n;
      s2 /= n;
#pragma unroll
      for (int k = 0; k < K; ++k)
#pragma unroll
        for (int e = 0; e < E; ++e) d[k][e] += (t[k][e] - s1 - h2[k][e] * s2) * rstd2;
    }
    s1 = s2 = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      float w[E], b[E];
      if (sh.after) w1_of.get(c.at, w);
      if (sh.gate == kRowGate && sh.after) b1_of.get(c.at, b);
      float out[E];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        out[e] = d[k][e] * sh.alpha;
        const float ee = d[k][e] * g[k][e];
        const float summed = sh.gate == kRowGate ? ee : d[k][e];
        sums[0][k][e] += summed * h1[k][e];
        sums[1][k][e] += summed;
        t[k][e] = sh.after ? ee * w[e] : ee;
        s1 += WHOLE || e >= c.own ? t[k][e] : 0.f;
        s2 += WHOLE || e >= c.own ? t[k][e] * h1[k][e] : 0.f;
      }
      if (!WHOLE && !c.live) continue;
      if (!sh.after) {
        put_pack<S, E>(dx + (r * sh.dim + c.at) * kS, out);
        put_pack<T, E>(df + (r * sh.dim + c.at) * kT, t[k]);
      }
      if (sh.gate == kRowGate) {
#pragma unroll
        for (int e = 0; e < E; ++e) out[e] = d[k][e] * (sh.after ? h1[k][e] * w[e] + b[e] : h1[k][e]);
        put_pack<T, E>(dgate + (r * sh.dim + c.at) * kT, out);
      }
    }
    if (!sh.after) continue;
    row_sums(s1, s2, lanes);
    s1 = sh.rms ? 0.f : s1 / n;
    s2 /= n;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const Columns<E> c(rows.lane + k * lanes, sh.dim);
      if (!WHOLE && !c.live) continue;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        t[k][e] = (t[k][e] - s1 - h1[k][e] * s2) * rstd1;
        d[k][e] *= sh.alpha;
      }
      // (dx, which may lie where dr does, behind the sums: all of the row has been read then, by all of its lanes)
      put_pack<S, E>(dx + (r * sh.dim + c.at) * kS, d[k]);
      put_pack<T, E>(df + (r * sh.dim + c.at) * kT, t[k]);
    }
  }
  if (part == nullptr) return;
  float* to = part + (int64_t)blockIdx.x * 4 * sh.dim;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const Columns<E> c(rows.lane + k * lanes, sh.dim);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (q < 2 ? !sh.after && sh.gate != kColumnGate : !sh.before) continue;  // (nobody reads these)
      if constexpr (WAVES == 1) {  // the block's groups have the same columns: the first adds up all of them
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e) lds[e * kBlock + threadIdx.x] = sums[q][k][e];
        __syncthreads();
        if (rows.group == 0)
          for (int i = 1; i < kBlock >> sh.lanes_log2; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) sums[q][k][e] += lds[e * kBlock + (i << sh.lanes_log2) + rows.lane];
      }
      if (rows.group == 0)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (e >= c.own) to[(int64_t)q * sh.dim + c.at + e] = sums[q][k][e];
    }
  }
}

// What the sums over the blocks' parts are: 64 columns a block, blockIdx.y the norm; its waves deal the blocks among themselves.
struct SeamGradients { float *dgate, *dw1, *db1, *dw2, *db2; };
constexpr int kSeamJoinWaves = 16;
template <int T>
__global__ __launch_bounds__(kSeamJoinWaves* kWave) void k_seam_join(const float* __restrict__ part, int blocks, SeamWeightPointers wp, SeamShape sh, SeamGradients out) {
  __shared__ float lds[2][kSeamJoinWaves][kWave];
  const int64_t c = (int64_t)blockIdx.x * kWave + lane_id();
  const bool second = blockIdx.y == 1;
  const float* from = part + (second ? 2 : 0) * (int64_t)sh.dim;
  float a = 0.f, b = 0.f;
  if (c < sh.dim) {
#pragma unroll 8
    for (int i = wave_in_block(); i < blocks; i += kSeamJoinWaves) {
      a += from[i * 4 * (int64_t)sh.dim + c];
      b += from[i * 4 * (int64_t)sh.dim + sh.dim + c];
    }
  }
  lds[0][wave_in_block()][lane_id()] = a;
  lds[1][wave_in_block()][lane_id()] = b;
  __syncthreads();
  if (wave_in_block() != 0 || c >= sh.dim) return;
  a = b = 0.f;
#pragma unroll
  for (int w = 0; w < kSeamJoinWaves; ++w) a += lds[0][w][lane_id()], b += lds[1][w][lane_id()];
  if (second) {
    if (out.dw2 != nullptr) out.dw2[c] = a;
    if (out.db2 != nullptr) out.db2[c] = b;
    return;
  }
  const auto value = [&](const char* p, float other) {
    return p == nullptr ? other : sh.wide_w ? ((const float*)p)[c] : (float)((const typename Element<T>::M*)p)[c];
  };
  const float g = sh.gate == kColumnGate ? value(wp.gate, 1.f) : 1.f;
  if (out.dw1 != nullptr) out.dw1[c] = g * a;
  if (out.db1 != nullptr) out.db1[c] = g * b;
  if (out.dgate != nullptr) out.dgate[c] = sh.after ? value(wp.w1, 1.f) * a + value(wp.b1, 0.f) * b : a;
}

constexpr int kLdsPiece = 1280;  // what a block's LDS is a multiple of

// How a row is shared: a pack a lane on one wave or less, on 2, 4 or 8 waves, and wider ones 2 or 4 packs a lane on 8.  (A pack a lane, for the
// registers: what a gradient holds for each column is 4 sums and 5 values besides the next row's.)
struct SeamLayout { int e, k, waves, lanes, lanes_log2; };
bool seam_layout(int32_t dim, int dtype, SeamLayout* out) {
  const int e = dtype == COOP_F32 ? 4 : 8;
  SeamLayout l{dim >= e ? e : 1, 1, 1, 1, 0};
  const int32_t packs = (dim + l.e - 1) / l.e;
  while (l.lanes < packs && l.lanes < 8 * kWave) l.lanes *= 2, ++l.lanes_log2;
  if (l.lanes > kWave) l.waves = l.lanes / kWave;
  while (l.k * l.lanes < packs) l.k *= 2;
  *out = l;
  return l.k <= 4;
}

// Blocks of a CU, by its registers, and of a forward call by what its weights take of the LDS too.  (A gradient's blocks have more registers, and fit.  A grid for the
// registers alone takes a second round for what does not fit.  bf16, a gate for each column and all weights and biases: 32,768 rows of 2,048 141 us, for 109, 65,536 of
// 1,024 157, for 108; 16,384 of 4,096 142, one block a CU 136, and with the last bias from memory two, 110.)
int64_t seam_resident(const SeamLayout& l, bool grad, int weights) {
  const int64_t most = 4 * seam_waves(l.e, l.k, l.waves, grad) / (l.waves == 1 ? kWavesPerBlock : l.waves);
  if (grad) return most;
  const int64_t fit = 160 * 1024 / ((weights + 16 * l.waves + kLdsPiece - 1) / kLdsPiece * kLdsPiece);
  return fit < most ? fit : most;
}
// Blocks of a pass: as many as are on the chip at once, and for a gradient no more
// than leave each group two rows.
int64_t seam_blocks(int64_t rows, const SeamLayout& l, bool grad, int weights = 0) {
  const int64_t per_block = l.waves == 1 ? kBlock / l.lanes : 1;
  int64_t b = (rows + per_block - 1) / per_block;
  const int64_t most = 256 * seam_resident(l, grad, weights);
  if (b > most) b = most;
  if (grad && b > rows / (2 * per_block) + 1) b = rows / (2 * per_block) + 1;
  return b;
}

template <int T, typename F>
void with_seam_layout(const SeamLayout& l, int32_t dim, F&& f) {
  constexpr int E = T == COOP_F32 ? 4 : 8;
  const auto call = [&](auto e, auto k, auto waves) {
    constexpr int EE = decltype(e)::value, K = decltype(k)::value;
    if (dim == EE * K * l.lanes) f(e, k, waves, std::integral_constant<bool, true>());
    else f(e, k, waves, std::integral_constant<bool, false>());
  };
  const std::integral_constant<int, E> wide;
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, 4> four;
  const std::integral_constant<int, 8> eight;
  if (l.e == 1) call(one, one, one);
  else if (l.waves == 1) call(wide, one, one);
  else if (l.waves == 2) call(wide, one, two);
  else if (l.waves == 4) call(wide, one, four);
  else l.k == 1 ? call(wide, one, eight) : l.k == 2 ? call(wide, two, eight) : call(wide, four, eight);
}
template <typename F>
void with_seam_types(int dtype, int stream_dtype, F&& f) {
  with_dtype(dtype, [&](auto t) {
    constexpr int T = decltype(t)::value;
    if (stream_dtype == COOP_F32) f(std::integral_constant<int, T>(), std::integral_constant<int, COOP_F32>());
    else if constexpr (T != COOP_F32) f(std::integral_constant<int, T>(), std::integral_constant<int, T>());
  });
}

constexpr int kNormFlags = COOP_NORM_AFTER | COOP_NORM_BEFORE | COOP_NORM_RMS;

int seam_check(int64_t rows, int32_t dim, int dtype, int stream_dtype, int weight_dtype, int norms, int gate_form, SeamLayout* l) {
  if (!known_dtype(dtype) || (stream_dtype != COOP_F32 && stream_dtype != dtype) || (weight_dtype != COOP_F32 && weight_dtype != dtype)) return COOP_E_ARG;
  if ((norms & ~kNormFlags) != 0 || (norms & (COOP_NORM_AFTER | COOP_NORM_BEFORE)) == 0) return COOP_E_ARG;
  if (rows < 0 || dim < 1 || !seam_layout(dim, dtype, l)) return COOP_E_ARG;
  if (gate_form != COOP_GATE_NONE && gate_form != COOP_GATE_COLUMNS && gate_form != COOP_GATE_ELEMENTS) return COOP_E_ARG;
  return COOP_OK;
}
SeamShape seam_shape(int64_t rows, int32_t dim, const SeamLayout& l, float alpha, float eps, int norms, int gate_form, int weight_dtype) {
  return SeamShape{rows, dim, l.lanes, l.lanes_log2, eps, alpha, (norms & COOP_NORM_AFTER) != 0, (norms & COOP_NORM_BEFORE) != 0, (norms & COOP_NORM_RMS) != 0,
                   gate_form, weight_dtype == COOP_F32, true};
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" int coop_residual_norm(const void* x, const void* f, int64_t n_rows, int32_t dim, int dtype, int stream_dtype, const void* gate,
                                  int gate_form, float alpha, int norms, const void* after_weight, const void* after_bias, const void* before_weight,
                                  const void* before_bias, int weight_dtype, float eps, void* r_out, void* y_out, float* stats_out, void* stream) {
  SeamLayout l;
  const int rc = seam_check(n_rows, dim, dtype, stream_dtype, weight_dtype, norms, gate_form, &l);
  if (rc != COOP_OK) return rc;
  const bool after = (norms & COOP_NORM_AFTER) != 0, before = (norms & COOP_NORM_BEFORE) != 0, rms = (norms & COOP_NORM_RMS) != 0;
  if (!(eps >= 0.f) || (rms && (after_bias || before_bias)) || (!after && (after_weight || after_bias)) || (!before && (before_weight || before_bias)))
    return COOP_E_ARG;
  if ((gate != nullptr) != (gate_form != COOP_GATE_NONE) && n_rows > 0) return COOP_E_ARG;
  if (n_rows == 0) return COOP_OK;
  if (!x || !f || !r_out || (before && !y_out) || !stats_out) return COOP_E_NULL;
  if (!aligned_for(x, stream_dtype) || !aligned_for(r_out, stream_dtype) || !aligned_for(f, dtype) || !aligned_for(y_out, dtype)) return COOP_E_ARG;
  for (const void* p : {after_weight, after_bias, before_weight, before_bias})
    if (!aligned_for(p, weight_dtype)) return COOP_E_ARG;
  if (gate && !aligned_for(gate, gate_form == COOP_GATE_COLUMNS ? weight_dtype : dtype)) return COOP_E_ARG;
  if (((uintptr_t)stats_out & 3) != 0) return COOP_E_ARG;
  SeamShape sh = seam_shape(n_rows, dim, l, alpha, eps, norms, gate_form, weight_dtype);
  const SeamWeightPointers wp{(const char*)gate, (const char*)after_weight, (const char*)after_bias, (const char*)before_weight, (const char*)before_bias};
  int weights = seam_lds(wp, gate_form == COOP_GATE_COLUMNS, dim);
  if (before_bias && weights > 0) {  // (a block would be alone on its CU for the last of its vectors: that is read from memory)
    const int without = weights - ((dim + 3) & ~3) * 4;
    if (seam_resident(l, false, weights) == 1 && seam_resident(l, false, without) > 1) weights = without, sh.last_in_lds = false;
  }
  const dim3 grid((unsigned)seam_blocks(n_rows, l, false, weights));
  with_seam_types(dtype, stream_dtype, [&](auto t, auto st) {
    constexpr int T = decltype(t)::value, S = decltype(st)::value;
    with_seam_layout<T>(l, dim, [&](auto e, auto k, auto waves, auto whole) {
      constexpr int E = decltype(e)::value, K = decltype(k)::value, N = decltype(waves)::value;
      const auto kernel = k_seam<T, S, E, K, N, decltype(whole)::value>;
      if (weights > 64 * 1024 - 512) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, weights);
      COOP_LAUNCH(K_SEAM, kernel, grid, dim3(kNormBlock<N>), weights, (hipStream_t)stream, (const char*)x, (const char*)f, wp, sh, (char*)r_out,
                  (char*)y_out, stats_out);
    });
  });
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_residual_norm_grad_workspace_bytes(int64_t n_rows, int32_t dim, int dtype) {
  SeamLayout l;
  if (seam_check(n_rows, dim, dtype, dtype, dtype, COOP_NORM_AFTER, COOP_GATE_NONE, &l) != COOP_OK) return 0;
  return (size_t)seam_blocks(n_rows, l, true) * 4 * (size_t)dim * sizeof(float) + 256;
}

extern "C" int coop_residual_norm_grad(const void* dr, const void* dy, const void* x, const void* f, int64_t n_rows, int32_t dim, int dtype, int stream_dtype,
                                       const float* stats, const void* gate, int gate_form, float alpha, int norms, const void* after_weight,
                                       const void* after_bias, const void* before_weight, int weight_dtype, void* dx, void* df, void* dgate,
                                       float* dafter_weight, float* dafter_bias, float* dbefore_weight, float* dbefore_bias, void* workspace,
                                       size_t workspace_bytes, void* stream) {
  SeamLayout l;
  const int rc = seam_check(n_rows, dim, dtype, stream_dtype, weight_dtype, norms, gate_form, &l);
  if (rc != COOP_OK) return rc;
  const bool after = (norms & COOP_NORM_AFTER) != 0, before = (norms & COOP_NORM_BEFORE) != 0, rms = (norms & COOP_NORM_RMS) != 0;
  if ((rms && after_bias) || (!after && (after_weight || after_bias || dafter_weight || dafter_bias)) || (!before && (before_weight || dbefore_weight || dbefore_bias)))
    return COOP_E_ARG;
  if (rms && (dafter_bias || dbefore_bias)) return COOP_E_ARG;
  // (of no elements gate and dgate have no address)
  if (gate_form != COOP_GATE_ELEMENTS || n_rows > 0)
    if ((gate != nullptr) != (gate_form != COOP_GATE_NONE) || (dgate != nullptr) != (gate_form != COOP_GATE_NONE)) return COOP_E_ARG;
  const SeamShape sh = seam_shape(n_rows, dim, l, alpha, 0.f, norms, gate_form, weight_dtype);
  if (n_rows > 0 && (!f || (before && (!dy || !x)) || (!before && !dr) || !stats || !dx || !df)) return COOP_E_NULL;
  const bool sums = dafter_weight || dafter_bias || dbefore_weight || dbefore_bias || sh.gate == kColumnGate;
  if (sums && !workspace) return COOP_E_NULL;
  for (const void* p : {dr, x, (const void*)dx})
    if (!aligned_for(p, stream_dtype)) return COOP_E_ARG;
  for (const void* p : {dy, f, (const void*)df})
    if (!aligned_for(p, dtype)) return COOP_E_ARG;
  for (const void* p : {after_weight, after_bias, before_weight})
    if (!aligned_for(p, weight_dtype)) return COOP_E_ARG;
  if (gate && (!aligned_for(gate, sh.gate == kColumnGate ? weight_dtype : dtype) || !aligned_for(dgate, sh.gate == kColumnGate ? COOP_F32 : dtype))) return COOP_E_ARG;
  for (const void* p : {(const void*)stats, (const void*)dafter_weight, (const void*)dafter_bias, (const void*)dbefore_weight, (const void*)dbefore_bias})
    if (((uintptr_t)p & 3) != 0) return COOP_E_ARG;
  if (sums && (workspace_bytes < coop_residual_norm_grad_workspace_bytes(n_rows, dim, dtype) || ((uintptr_t)workspace & 15) != 0)) return COOP_E_ARG;
  const hipStream_t s = (hipStream_t)stream;
  const SeamWeightPointers wp{(const char*)gate, (const char*)after_weight, (const char*)after_bias, (const char*)before_weight, nullptr};
  const int64_t blocks = seam_blocks(n_rows, l, true);
  const int weights = seam_lds(wp, gate_form == COOP_GATE_COLUMNS, dim);
  float* part = sums ? (float*)workspace : nullptr;
  if (n_rows > 0)
    with_seam_types(dtype, stream_dtype, [&](auto t, auto st) {
      constexpr int T = decltype(t)::value, S = decltype(st)::value;
      with_seam_layout<T>(l, dim, [&](auto e, auto k, auto waves, auto whole) {
        constexpr int E = decltype(e)::value, K = decltype(k)::value, N = decltype(waves)::value;
        const auto kernel = k_seam_grad<T, S, E, K, N, decltype(whole)::value>;
        if (weights > 64 * 1024 - 8192) (void)hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, weights);
        COOP_LAUNCH(K_SEAM_GRAD, kernel, dim3((unsigned)blocks), dim3(kNormBlock<N>), weights, s, (const char*)dr, (const char*)dy,
                    (const char*)x, (const char*)f, stats, wp, sh, (char*)dx, (char*)df, (char*)dgate, part);
      });
    });
  if (sums) {
    const SeamGradients out{sh.gate == kColumnGate ? (float*)dgate : nullptr, dafter_weight, dafter_bias, dbefore_weight, dbefore_bias};
    with_dtype(dtype, [&](auto t) {
      COOP_LAUNCH(K_SEAM_JOIN, k_seam_join<decltype(t)::value>, dim3((unsigned)((dim + kWave - 1) / kWave), before ? 2 : 1), dim3(kSeamJoinWaves * kWave), 0, s,
                  (const float*)part, n_rows > 0 ? (int)blocks : 0, wp, sh, out);
    });
  }
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
