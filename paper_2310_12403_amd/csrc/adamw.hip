// AdamW over many tensors, or over the touched rows of a table, in one pass: with g the gradient (times *grad_scale),
//   m <- beta1 m + (1 - beta1) g,   v <- beta2 v + (1 - beta2) g^2,
//   p <- p (1 - lr wd) - lr (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps).
//
// Bound by HBM: parameter, gradient and moments are read once and written once.  All arithmetic is in 32 bits; every product and sum
// is rounded on its own (the file is compiled without contraction).
// 300 tensors, 100 million parameters in fp32, gradients and copies in bf16: 545 us, 2.8 GB at 5.1 TB/s.  500,000 of 2.45 million rows of
// 100 parameters, moments in 8 bits: 279 us for 0.8 GB, 1.07 GB with the whole 128-byte lines of rows of 400 and of 100 bytes.
//
// Moments in 8 bits.  m, and the root of v (half the exponents, and never negative), are kept as 8-bit floats of 4 exponent and 3
// mantissa bits (OCP E4M3) over a 32-bit scale for each 256 neighbouring elements of a row: scale = largest magnitude / 448, so the
// smallest number that is not lost is 2^-17.8 of the block's largest.  Neighbouring numbers lie 6 to 12 % apart: rounded to the nearest, a
// decay of 0.1 % a step would never be seen, and v could not leave its value until g^2 were dozens of times as large.  So they are
// rounded up or down at random with the mean at the value itself; the random number is a hash of (seed, step, tensor, element), the
// same on every run.  A root that is not zero is never rounded to zero, or a parameter whose gradient stops would be divided by eps.
// With y the value over its scale, the bits of the 32-bit float 2^-120 |y| are exponent and mantissa of the 8-bit one and 20 bits below
// them, E4M3's subnormals included: adding 20 random bits and cutting them off is the rounding.
// A moment that is not finite makes its block's scale NaN or infinite, and so all of the block's moments; blocks whose largest is below
// 2^-117 are kept as zeros.
#include <type_traits>

#include "coop_internal.h"
#include "elements.h"
#include "variates.h"

namespace coop {
namespace {

constexpr int kMomentBlock = 256;  // elements that share a scale: 4 neighbouring ones for each lane of a wave.  Rows of up to 128 (64, 32)
                                   // elements are a block each and take 32 (16, 8) lanes, two or more to a wave.
constexpr int kPerLane = 4;
constexpr int kBlocksPerWave = 4;
constexpr int kBlocksPerGroup = kWavesPerBlock * kBlocksPerWave;
constexpr int64_t kMostGroups = (int64_t)1 << 23;  // of a tensor: with those in front of it in its launch fewer than 2^32 threads

int lanes_log2_of(int64_t dim) { return dim <= 32 ? 3 : dim <= 64 ? 4 : dim <= 128 ? 5 : 6; }
int64_t groups_of(int64_t blocks, int lanes_log2) {
  const int64_t per_group = (int64_t)kBlocksPerGroup << (6 - lanes_log2);
  return (blocks + per_group - 1) / per_group;
}

// What every tensor needs, and what only 8-bit moments or listed rows do.
struct Whole {
  char *param, *copy, *m, *v;
  const char* grad;
  int64_t dim;
  uint32_t row_blocks;   // blocks of 256 elements per row, the last one of what is left
  uint32_t n_blocks;     // of all rows, or of as many rows as the list may have
  uint32_t first_group;  // of the launch's thread blocks
  uint8_t lanes_log2;    // lanes for a block: 64, or fewer that hold all of a row
  int8_t param_type, grad_type, copy_type;
};
struct Listed : Whole {
  float *m_scale, *v_scale;
  const int32_t *rows, *n_active;
  int64_t n_rows;
  uint32_t key[4];
};

struct Hyper { float keep1, take1, keep2, take2, decay, rate, undo, eps; };

// A launch's tensors are its arguments (at most 4 KB): nothing is copied to the device ahead of it, and nothing is kept.  (62 tensors
// with 32-bit moments and without a list: 300 of them in 5 launches in the place of 12, 647 -> 558 us with non-temporal accesses.)
template <typename Tensor>
struct Step {
  static constexpr int kTensors = (4096 - 72) / (int)sizeof(Tensor);
  Hyper h;
  int n;
  int32_t* bad;
  const float* grad_scale;
  Tensor t[kTensors];
};
static_assert(sizeof(Step<Whole>) <= 4096 && sizeof(Step<Listed>) <= 4096, "kernel arguments");

// Elements i .. i + 3 of an array of the type, those beyond n as zero
__device__ __forceinline__ void load4(const char* p, int type, int64_t i, int n, float (&f)[4]) {
  if (n >= 4) {
    if (type == COOP_F32) Pack<COOP_F32, 4>::load_nt(p + i * 4).get(f);
    else if (type == COOP_F16) Pack<COOP_F16, 4>::load_nt(p + i * 2).get(f);
    else Pack<COOP_BF16, 4>::load_nt(p + i * 2).get(f);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = 0.f;
    if (e < n) f[e] = type == COOP_F32 ? ((const float*)p)[i + e] : type == COOP_F16 ? (float)((const _Float16*)p)[i + e] : (float)((const __bf16*)p)[i + e];
  }
}
__device__ __forceinline__ void store4(char* p, int type, int64_t i, int n, const float (&f)[4]) {
  if (n >= 4) {
    if (type == COOP_F32) { Pack<COOP_F32, 4> x; x.set(f); x.store_nt(p + i * 4); }
    else if (type == COOP_F16) { Pack<COOP_F16, 4> x; x.set(f); x.store_nt(p + i * 2); }
    else { Pack<COOP_BF16, 4> x; x.set(f); x.store_nt(p + i * 2); }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) {
      if (type == COOP_F32) ((float*)p)[i + e] = f[e];
      else if (type == COOP_F16) ((_Float16*)p)[i + e] = (_Float16)f[e];
      else ((__bf16*)p)[i + e] = (__bf16)f[e];
    }
}
typedef uint32_t u32_any __attribute__((aligned(1)));
__device__ __forceinline__ uint32_t load_codes(const char* p, int n) {
  if (n >= 4) return *reinterpret_cast<const u32_any*>(p);
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) c |= (uint32_t)(uint8_t)p[e] << (8 * e);
  return c;
}
__device__ __forceinline__ void store_codes(char* p, int n, uint32_t c) {
  if (n >= 4) { *reinterpret_cast<u32_any*>(p) = c; return; }
#pragma unroll
  for (int e = 0; e < 3; ++e)
    if (e < n) p[e] = (char)(c >> (8 * e));
}

__device__ __forceinline__ float code_value(uint32_t code) {  // of the 8-bit float
  const float a = __uint_as_float((code & 0x7Fu) << 20) * 0x1p120f;
  const float x = (code & 0x7Fu) == 0x7Fu ? __uint_as_float(0x7FC00000u) : a;
  return code & 0x80u ? -x : x;
}

// The four codes of a lane; scale: of its block.  `floor`: the code of a value that is not zero is at least this.  The quotients are
// the reciprocal's, made exact by one step: an ulp more or less could take a value over the bound between two codes.
__device__ __forceinline__ uint32_t encode(const float (&x)[4], float scale, const uint32_t (&noise)[4], uint32_t floor) {
  float by = __builtin_amdgcn_rcpf(scale);
  by = __builtin_fmaf(__builtin_fmaf(-scale, by, 1.f), by, by);
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float q = x[e] * by, y = __builtin_fmaf(__builtin_fmaf(-q, scale, x[e]), by, q);
    const uint32_t bits = __float_as_uint(fabsf(y) * 0x1p-120f);
    uint32_t code = (bits + noise[e]) >> 20;
    code = code < 0x7Eu ? code : 0x7Eu;
    if (code == 0) code = floor;
    if (x[e] == 0.f || scale == 0.f) code = 0;
    if (x[e] < 0.f) code |= 0x80u;
    c |= code << (8 * e);
  }
  return c;
}
// The scale of a block that `lanes` lanes share.  A NaN counts as larger than any number; below 2^-126 (its reciprocal would not be a
// number) the block is taken as zeros.
__device__ __forceinline__ float block_scale(const float (&x)[4], int lanes) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t b = __float_as_uint(x[e]) & 0x7FFFFFFFu;
    top = top > b ? top : b;
  }
  for (int off = 1; off < lanes; off <<= 1) {
    const uint32_t o = __shfl_xor(top, off, kWave);
    top = top > o ? top : o;
  }
  const float scale = __uint_as_float(top) * (1.f / 448.f);
  return scale < 0x1p-126f ? 0.f : scale;
}

template <int BITS, typename Tensor>
__global__ __launch_bounds__(kBlock) void k_adamw(Step<Tensor> st) {
  constexpr bool kListed = std::is_same<Tensor, Listed>::value;
  // the tensor that this block belongs to: the last one that begins at or before it
  int lo = 0, hi = st.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (st.t[mid].first_group <= blockIdx.x) lo = mid;
    else hi = mid;
  }
  const Tensor& t = st.t[lo];
  const float gs = st.grad_scale != nullptr ? *st.grad_scale : 1.f;
  int32_t active = 0x7FFFFFFF;
  if constexpr (kListed)
    if (t.n_active != nullptr) active = *t.n_active;
  const int lanes = 1 << t.lanes_log2, lane = lane_id() & (lanes - 1);
  const uint32_t each = kWave >> t.lanes_log2;  // blocks that a wave has at a time
#pragma unroll 1
  for (int q = 0; q < kBlocksPerWave; ++q) {
    const uint32_t b = ((blockIdx.x - t.first_group) * kBlocksPerGroup + q * kWavesPerBlock + uniform_wave_in_block()) * each;
    uint32_t entry, in_row;
    if (each == 1) {
      entry = b / t.row_blocks;
      in_row = b - entry * t.row_blocks;
    } else {
      entry = b + (lane_id() >> t.lanes_log2);
      in_row = 0;
    }
    if (b >= t.n_blocks) return;
    int64_t row = entry;
    bool there = each == 1 || entry < t.n_blocks;
    if constexpr (kListed)
      if (t.rows != nullptr) {
        there = there && (int32_t)entry < active;
        row = there ? t.rows[entry] : 0;
        if ((uint64_t)row >= (uint64_t)t.n_rows) {
          if (lane == 0 && in_row == 0) atomicOr(st.bad, 1);
          there = false;
        }
      }
    if (!there) continue;
    const int64_t col = (int64_t)in_row * kMomentBlock + lane * kPerLane, left = t.dim - col;
    const int n = left < 0 ? 0 : left < 4 ? (int)left : 4;
    const int64_t at = row * t.dim + col, grad_at = (int64_t)entry * t.dim + col;
    const int64_t scale_at = row * t.row_blocks + in_row;
    float p[4], g[4], m[4], v[4], root[4];
    load4(t.grad, t.grad_type, grad_at, n, g);
    load4(t.param, t.param_type, at, n, p);
    if constexpr (BITS == 32) {
      load4(t.m, COOP_F32, at, n, m);
      load4(t.v, COOP_F32, at, n, v);
    } else {
      const uint32_t mc = load_codes(t.m + at, n), vc = load_codes(t.v + at, n);
      const float ms = t.m_scale[scale_at], vs = t.v_scale[scale_at];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        m[e] = code_value(mc >> (8 * e) & 0xFFu) * ms;
        root[e] = code_value(vc >> (8 * e) & 0xFFu) * vs;
        v[e] = root[e] * root[e];
        if (e >= n) m[e] = v[e] = 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (st.grad_scale != nullptr) g[e] *= gs;
      m[e] = m[e] * st.h.keep1 + g[e] * st.h.take1;
      v[e] = v[e] * st.h.keep2 + (g[e] * g[e]) * st.h.take2;
      root[e] = sqrtf(v[e]);
      if constexpr (BITS == 32) p[e] = p[e] * st.h.decay - (m[e] / (root[e] * st.h.undo + st.h.eps)) * st.h.rate;
      else p[e] = p[e] * st.h.decay - (m[e] * __builtin_amdgcn_rcpf(root[e] * st.h.undo + st.h.eps)) * st.h.rate;  // (moments of four bits)
      if (e >= n) m[e] = root[e] = 0.f;
    }
    store4(t.param, t.param_type, at, n, p);
    if (t.copy != nullptr) store4(t.copy, t.copy_type, at, n, p);
    if constexpr (BITS == 32) {
      store4(t.m, COOP_F32, at, n, m);
      store4(t.v, COOP_F32, at, n, v);
    } else {
      const float ms = block_scale(m, lanes), vs = block_scale(root, lanes);
      const uint64_t element = ((uint64_t)row * t.row_blocks + in_row) * kMomentBlock + (uint32_t)(lane * kPerLane);
      // u = mix(mix(low ^ key0) ^ key1 ^ mix(high ^ key2)) ^ key3 of the element's number.  A block's elements share the high word, and a
      // lane's the low one but for its last two bits; the fold that ends the inner mixer and the one that begins the outer cancel.
      const uint32_t high = fold16(mix32((uint32_t)(element >> 32) ^ t.key[2]) ^ t.key[1]), low = (uint32_t)element ^ t.key[0];
      uint32_t nm[4], nv[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t u = fold16_xor(mix_body(mix_body(fold16(low ^ (uint32_t)e)) ^ high), t.key[3]);
        nm[e] = ((u & 0xFFFFu) << 4) + 8;  // 16 random bits each, in the middle of the 16 values they stand for
        nv[e] = (u >> 16 << 4) + 8;
      }
      const uint32_t mc = encode(m, ms, nm, 0u), vc = encode(root, vs, nv, 1u);
      store_codes(t.m + at, n, mc);
      store_codes(t.v + at, n, vc);
      if (lane == 0) {
        t.m_scale[scale_at] = ms;
        t.v_scale[scale_at] = vs;
      }
    }
  }
}

template <int BITS, typename Tensor>
void launch_steps(const coop_adamw_tensor* tensors, int n, const Hyper& h, int64_t step, uint64_t seed, const float* grad_scale, int32_t* bad,
                  hipStream_t s) {
  Step<Tensor> st;
  st.h = h;
  st.bad = bad;
  st.grad_scale = grad_scale;
  uint32_t groups = 0;
  st.n = 0;
  const auto flush = [&] {
    if (st.n > 0) COOP_LAUNCH(K_ADAMW, (k_adamw<BITS, Tensor>), dim3(groups), dim3(kBlock), 0, s, st);
    st.n = 0;
    groups = 0;
  };
  for (int i = 0; i < n; ++i) {
    const coop_adamw_tensor& t = tensors[i];
    const int64_t rows = t.rows ? t.n_list : t.n_rows;
    if (rows == 0 || t.dim == 0) continue;
    Tensor& d = st.t[st.n];
    d.param = (char*)t.param, d.copy = (char*)t.copy, d.m = (char*)t.m, d.v = (char*)t.v, d.grad = (const char*)t.grad;
    d.dim = t.dim;
    d.row_blocks = (uint32_t)((t.dim - 1) / kMomentBlock + 1);
    d.n_blocks = (uint32_t)(rows * d.row_blocks);
    d.first_group = groups;
    d.lanes_log2 = (uint8_t)lanes_log2_of(t.dim);
    d.param_type = (int8_t)t.param_dtype, d.grad_type = (int8_t)t.grad_dtype, d.copy_type = (int8_t)t.copy_dtype;
    if constexpr (std::is_same<Tensor, Listed>::value) {
      d.m_scale = t.m_scale, d.v_scale = t.v_scale, d.rows = t.rows, d.n_active = t.n_list_dev, d.n_rows = t.n_rows;
      const uint32_t ctr[4] = {(uint32_t)step, (uint32_t)((uint64_t)step >> 32), (uint32_t)i, 0x4144414Du};
      const uint32_t key[2] = {(uint32_t)seed, (uint32_t)(seed >> 32)};
      philox4x32_10(ctr, key, d.key);
    }
    groups += (uint32_t)groups_of(d.n_blocks, d.lanes_log2);
    if (++st.n == Step<Tensor>::kTensors || groups >= kMostGroups / 2) flush();
  }
  flush();
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" int coop_adamw(const coop_adamw_tensor* tensors, int n, int bits, double lr, double beta1, double beta2, double eps,
                          double weight_decay, int64_t step, uint64_t seed, const float* grad_scale, void* stream) {
  if (n < 0 || (bits != 32 && bits != 8) || step < 1) return COOP_E_ARG;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !(lr >= 0.0) || !(weight_decay >= 0.0)) return COOP_E_ARG;
  if (n == 0) return COOP_OK;
  if (!tensors) return COOP_E_NULL;
  for (int i = 0; i < n; ++i) {  // every tensor is looked at before the first launch
    const coop_adamw_tensor& t = tensors[i];
    if (!known_dtype(t.param_dtype) || !known_dtype(t.grad_dtype) || (t.copy && !known_dtype(t.copy_dtype))) return COOP_E_ARG;
    if (t.n_rows < 0 || t.dim < 0 || t.n_list < 0 || t.n_rows >= ((int64_t)1 << 31) || t.n_list >= ((int64_t)1 << 31)) return COOP_E_ARG;
    if (t.rows == nullptr && t.n_list_dev != nullptr) return COOP_E_ARG;
    const int64_t rows = t.rows ? t.n_list : t.n_rows;
    if (rows == 0 || t.dim == 0) continue;
    if (t.dim > INT64_MAX / 8 / (t.n_rows > 0 ? t.n_rows : 1)) return COOP_E_ARG;
    const int64_t row_blocks = (t.dim - 1) / kMomentBlock + 1;
    if (row_blocks > ((int64_t)1 << 27) || groups_of(rows * row_blocks, lanes_log2_of(t.dim)) > kMostGroups) return COOP_E_ARG;
    if (!t.param || !t.grad || !t.m || !t.v || (bits == 8 && (!t.m_scale || !t.v_scale))) return COOP_E_NULL;
    if (!aligned_for(t.param, t.param_dtype) || !aligned_for(t.grad, t.grad_dtype) || (t.copy && !aligned_for(t.copy, t.copy_dtype))) return COOP_E_ARG;
    if ((bits == 32 && (((uintptr_t)t.m | (uintptr_t)t.v) & 3) != 0) || (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3) != 0) return COOP_E_ARG;
  }
  bool listed = bits == 8;
  for (int i = 0; i < n; ++i) listed |= tensors[i].rows != nullptr;
  const Hyper h{(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)(1.0 - lr * weight_decay),
                (float)(lr / (1.0 - pow(beta1, (double)step))), (float)(1.0 / sqrt(1.0 - pow(beta2, (double)step))), (float)eps};
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  const hipStream_t s = (hipStream_t)stream;
  if (bits == 8) launch_steps<8, Listed>(tensors, n, h, step, seed, grad_scale, bad, s);
  else if (listed) launch_steps<32, Listed>(tensors, n, h, step, seed, grad_scale, bad, s);
  else launch_steps<32, Whole>(tensors, n, h, step, seed, grad_scale, bad, s);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}
