// The norm of all gradients and the factor that clips them, ahead of an optimizer's step: norm = |s| sqrt(sum over all tensors of g^2),
// factor = s min(1, max_norm / (norm + 1e-6)), with s a factor that the gradients are to be multiplied by anyway (a loss scale taken back).
//
// Bound by HBM: every gradient is read once.  Squares are added up in 64 bits, where those of numbers of 24 bits are exact, nothing overflows and
// nothing is lost, in an order that the sizes alone decide: a lane's, a block's, and then one block's over all of them.
#include <algorithm>
#include <memory>
#include <new>
#include <utility>

#include "coop_internal.h"
#include "elements.h"

namespace coop {
namespace {

constexpr int kPiece = 16384;  // elements that a block has at a time
constexpr int64_t kMostPieces = (int64_t)1 << 24;

struct Grad {
  char* p;
  int64_t n;             // elements
  uint32_t first_piece;  // of the launch's
  int16_t type;
  int16_t touched;       // -1: all of them; else which of the launch's counts says how many
};
struct Touched {
  const int32_t* rows;  // that many rows of dim elements
  int64_t dim;
};
struct Grads {
  static constexpr int kTouched = 16, kTensors = (4096 - 64 - kTouched * (int)sizeof(Touched)) / (int)sizeof(Grad);
  const float* factor;
  double* part;
  int n, n_touched;
  uint32_t pieces;
  Touched touched[kTouched];
  Grad t[kTensors];
};
static_assert(sizeof(Grads) <= 4096, "kernel arguments");

// The tensor that a piece belongs to, and the piece's elements.
struct Mine {
  const Grad* t;
  int64_t first, last;
  __device__ __forceinline__ Mine(const Grads& g, uint32_t piece) {
    int lo = 0, hi = g.n;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (g.t[mid].first_piece <= piece) lo = mid;
      else hi = mid;
    }
    t = &g.t[lo];
    int64_t n = t->n;
    if (t->touched >= 0) {
      const Touched& of = g.touched[t->touched];
      const int64_t there = *of.rows * of.dim;
      n = there < n ? there < 0 ? 0 : there : n;
    }
    first = (int64_t)(piece - t->first_piece) * kPiece;
    last = first + kPiece < n ? first + kPiece : n;
  }
};

template <int T, typename F>
__device__ __forceinline__ void over(char* p, int64_t first, int64_t last, F&& f) {
  constexpr int E = 16 / (int)sizeof(typename Element<T>::M);
  typedef typename Element<T>::M M;
  if (last - first == kPiece) {  // (all of its loads are on their way at once)
#pragma unroll
    for (int i = 0; i < kPiece / (kBlock * E); ++i) f(std::integral_constant<int, E>(), (M*)p + first + (i * kBlock + (int)threadIdx.x) * E);
    return;
  }
  const int64_t whole = first + (last - first) / E * E;
#pragma unroll 4
  for (int64_t i = first + threadIdx.x * E; i < whole; i += kBlock * E) f(std::integral_constant<int, E>(), (M*)p + i);
  for (int64_t i = whole + threadIdx.x; i < last; i += kBlock) f(std::integral_constant<int, 1>(), (M*)p + i);
}

template <typename F>
__device__ __forceinline__ void over_any(const Grad& t, int64_t first, int64_t last, F&& f) {
  if (t.type == COOP_F32) over<COOP_F32>(t.p, first, last, [&](auto e, auto* p) { f(std::integral_constant<int, COOP_F32>(), e, p); });
  else if (t.type == COOP_F16) over<COOP_F16>(t.p, first, last, [&](auto e, auto* p) { f(std::integral_constant<int, COOP_F16>(), e, p); });
  else over<COOP_BF16>(t.p, first, last, [&](auto e, auto* p) { f(std::integral_constant<int, COOP_BF16>(), e, p); });
}

// part[block]: the squares of the block's pieces
__global__ __launch_bounds__(kBlock) void k_grad_norm(Grads g) {
  double sum = 0.0;
  for (uint32_t piece = blockIdx.x; piece < g.pieces; piece += gridDim.x) {
    const Mine mine(g, piece);
    over_any(*mine.t, mine.first, mine.last, [&](auto t, auto e, auto* p) {
      constexpr int T = decltype(t)::value, E = decltype(e)::value;
      float x[E];
      Pack<T, E>::load_nt(p).get(x);
#pragma unroll
      for (int i = 0; i < E; ++i) sum = __builtin_fma((double)x[i], (double)x[i], sum);
    });
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) sum += __shfl_xor(sum, off, kWave);
  __shared__ double lds[kWavesPerBlock];
  if (lane_id() == 0) lds[wave_in_block()] = sum;
  __syncthreads();
  if (threadIdx.x == 0) g.part[blockIdx.x] = (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

__global__ __launch_bounds__(1024) void k_grad_factor(const double* __restrict__ part, int n, const float* __restrict__ scale, double max_norm,
                                                      float* __restrict__ norm_out, float* __restrict__ factor_out) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) sum += part[i];
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) sum += __shfl_xor(sum, off, kWave);
  __shared__ double lds[16];
  if (lane_id() == 0) lds[wave_in_block()] = sum;
  __syncthreads();
  if (threadIdx.x != 0) return;
  sum = 0.0;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += lds[w];
  const double s = scale != nullptr ? (double)*scale : 1.0, norm = fabs(s) * sqrt(sum);
  const double over = norm < __builtin_inf() || norm != norm ? max_norm / (norm + 1e-6) : 0.0;  // (an infinite norm is above any bound, an infinite one too)
  if (norm_out != nullptr) *norm_out = (float)norm;
  if (factor_out != nullptr) *factor_out = (float)(over >= 1.0 ? s : s * over);  // (of a norm that is no number: no number)
}

__global__ __launch_bounds__(kBlock) void k_grad_scale(Grads g) {
  const float factor = *g.factor;
  if (factor == 1.f) return;  // (as most steps have it that are not clipped)
  for (uint32_t piece = blockIdx.x; piece < g.pieces; piece += gridDim.x) {
    const Mine mine(g, piece);
    over_any(*mine.t, mine.first, mine.last, [&](auto t, auto e, auto* p) {
      constexpr int T = decltype(t)::value, E = decltype(e)::value;
      float x[E];
      Pack<T, E> v = Pack<T, E>::load_nt(p);
      v.get(x);
#pragma unroll
      for (int i = 0; i < E; ++i) x[i] *= factor;
      v.set(x);
      v.store_nt(p);
    });
  }
}

constexpr uint32_t kMostBlocks = 2048;
uint32_t blocks_of(uint32_t pieces) { return pieces < kMostBlocks ? pieces : kMostBlocks; }

// f(grads, blocks) for every launch
template <typename F>
void in_launches(const coop_grad_tensor* tensors, int n, F&& f) {
  Grads g;
  g.factor = nullptr;
  g.part = nullptr;
  g.n = g.n_touched = 0;
  g.pieces = 0;
  const auto flush = [&] {
    if (g.n > 0) f(g, blocks_of(g.pieces));
    g.n = g.n_touched = 0;
    g.pieces = 0;
  };
  for (int i = 0; i < n; ++i) {
    const coop_grad_tensor& t = tensors[i];
    if (t.n_rows == 0 || t.dim == 0) continue;
    const int64_t count = t.n_rows * t.dim;
    if (t.n_rows_dev != nullptr) g.touched[g.n_touched] = Touched{t.n_rows_dev, t.dim};
    g.t[g.n++] = Grad{(char*)t.grad, count, g.pieces, (int16_t)t.dtype, (int16_t)(t.n_rows_dev != nullptr ? g.n_touched++ : -1)};
    g.pieces += (uint32_t)((count + kPiece - 1) / kPiece);
    if (g.n == Grads::kTensors || g.n_touched == Grads::kTouched || g.pieces >= kMostPieces) flush();
  }
  flush();
}

int grads_check(const coop_grad_tensor* tensors, int n) {
  if (n < 0) return COOP_E_ARG;
  if (n > 0 && !tensors) return COOP_E_NULL;
  for (int i = 0; i < n; ++i) {
    const coop_grad_tensor& t = tensors[i];
    if (!known_dtype(t.dtype) || t.n_rows < 0 || t.dim < 0) return COOP_E_ARG;
    if (t.n_rows == 0 || t.dim == 0) continue;
    if (t.dim > (kMostPieces * kPiece) / t.n_rows) return COOP_E_ARG;
    if (!t.grad) return COOP_E_NULL;
    if (!aligned_for(t.grad, t.dtype) || ((uintptr_t)t.n_rows_dev & 3) != 0) return COOP_E_ARG;
  }
  return COOP_OK;
}

// Whether no two of them have an element in common (COOP_OK): blocks that multiply the same one meet in memory.
int grads_apart(const coop_grad_tensor* tensors, int n) {
  typedef std::pair<uintptr_t, uintptr_t> Range;
  const std::unique_ptr<Range[]> at(new (std::nothrow) Range[(size_t)n]);
  if (!at) return COOP_E_NOMEM;
  int k = 0;
  for (int i = 0; i < n; ++i) {
    const uintptr_t p = (uintptr_t)tensors[i].grad;
    const int64_t count = tensors[i].n_rows * tensors[i].dim;
    if (count > 0) at[k++] = Range(p, p + (uintptr_t)count * (uintptr_t)element_bytes(tensors[i].dtype));
  }
  std::sort(at.get(), at.get() + k);
  for (int i = 1; i < k; ++i)
    if (at[i].first < at[i - 1].second) return COOP_E_ARG;
  return COOP_OK;
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" size_t coop_grad_norm_workspace_bytes(const coop_grad_tensor* tensors, int n) {
  if (grads_check(tensors, n) != COOP_OK) return 0;
  size_t blocks = 0;
  in_launches(tensors, n, [&](const Grads&, uint32_t b) { blocks += b; });
  return blocks * sizeof(double) + 256;
}

extern "C" int coop_grad_norm(const coop_grad_tensor* tensors, int n, double max_norm, const float* grad_scale, float* norm_out, float* factor_out,
                              void* workspace, size_t workspace_bytes, void* stream) {
  const int rc = grads_check(tensors, n);
  if (rc != COOP_OK) return rc;
  if (!(max_norm >= 0.0)) return COOP_E_ARG;
  if (!norm_out && !factor_out) return COOP_OK;
  if (!workspace) return COOP_E_NULL;
  if ((((uintptr_t)grad_scale | (uintptr_t)norm_out | (uintptr_t)factor_out) & 3) != 0) return COOP_E_ARG;
  if (((uintptr_t)workspace & 7) != 0 || workspace_bytes < coop_grad_norm_workspace_bytes(tensors, n)) return COOP_E_ARG;
  const hipStream_t s = (hipStream_t)stream;
  double* part = (double*)workspace;
  int parts = 0;
  in_launches(tensors, n, [&](Grads& g, uint32_t blocks) {
    g.part = part + parts;
    parts += (int)blocks;
    COOP_LAUNCH(K_GRAD_NORM, k_grad_norm, dim3(blocks), dim3(kBlock), 0, s, g);
  });
  COOP_LAUNCH(K_GRAD_FACTOR, k_grad_factor, dim3(1), dim3(1024), 0, s, (const double*)part, parts, grad_scale, max_norm, norm_out, factor_out);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" int coop_grad_scale(const coop_grad_tensor* tensors, int n, const float* factor, void* stream) {
  const int rc = grads_check(tensors, n);
  if (rc != COOP_OK) return rc;
  if (n == 0) return COOP_OK;
  if (!factor) return COOP_E_NULL;
  if (((uintptr_t)factor & 3) != 0) return COOP_E_ARG;
  const int apart = grads_apart(tensors, n);
  if (apart != COOP_OK) return apart;
  const hipStream_t s = (hipStream_t)stream;
  in_launches(tensors, n, [&](Grads& g, uint32_t blocks) {
    g.factor = factor;
    COOP_LAUNCH(K_GRAD_SCALE, k_grad_scale, dim3(blocks), dim3(kBlock), 0, s, g);
  });
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
