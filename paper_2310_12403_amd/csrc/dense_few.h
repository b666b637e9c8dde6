// Dense layers forward, of few rows (one token first of all) or small altogether: operands straight from memory, of any alignment, into the matrix
// units' registers, and one launch.  Included by dense.hip.
//
// A block has 16 columns by 32 rows of the result, so that there are blocks for every CU, and all of k: its waves deal it among themselves, 128
// bytes of a row at a time, and their sums meet in LDS.  Of few rows it is the weight that bounds it, and that is read once.  (4,096 x 4,096 in
// bf16, one row: 8.1 us; tiles with k dealt to blocks, and a second launch that joins them: 13.2.)
#pragma once

typedef float f32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of both operands into a 16 x 16 tile: a lane has row lane & 15 and a quarter of a step of k
template <int T>
__device__ __forceinline__ f32x4 mma16(u32x4 a, u32x4 b, f32x4 c) {
  if constexpr (T == COOP_F16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else if constexpr (T == COOP_BF16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
  }
}

constexpr int kFewRows = 32, kFewMany = 1024;  // bytes of a row from which on a block has 16 waves, of less 4: a wave has 128 bytes at least

// NT: tiles of 16 rows of x
// Fin: what becomes of the sums (Slope's columns: a part for every 16 rows)
template <int T, int NT, bool PAIR, int WAVES, typename Fin>
__global__ __launch_bounds__(WAVES* kWave) void k_few(const char* __restrict__ x, const char* __restrict__ w, const char* __restrict__ w2, int64_t n, int32_t k,
                                                           Fin fin) {
  typedef typename Element<T>::M M;
  constexpr int E = kE<T>, P = PAIR ? 2 : 1, kStep = 4 * E, kAhead = 2;  // elements of k in a step; pairs of steps on their way at a time
  __shared__ __attribute__((aligned(16))) float part[WAVES][P][NT * 16][16];
  const int wave = uniform_wave_in_block(), lane = lane_id(), r16 = lane & 15, quarter = lane >> 4;
  const int32_t col0 = (int32_t)blockIdx.x * 16;
  const int64_t row0 = (int64_t)blockIdx.y * kFewRows;
  const int32_t col = col0 + r16 < fin.cols ? col0 + r16 : fin.cols - 1;  // (what is not there: the last one's, and nothing is stored)
  const int64_t ld = (int64_t)k * kElem<T>;
  const char* const from_w[2] = {w + col * ld, PAIR ? w2 + col * ld : nullptr};
  const char* from_x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) from_x[t] = x + (row0 + t * 16 + r16 < n ? row0 + t * 16 + r16 : n - 1) * ld;
  f32x4 acc[P][NT];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = k / kStep;  // whole ones
  const auto chunk = [&](const char* row, int step) { return __builtin_bit_cast(u32x4, Pack<T, E>::load(row + (int64_t)step * 64 + quarter * 16)); };
  constexpr int kStride = WAVES * 2;
  for (int base = wave * 2; base < steps; base += kStride * kAhead) {
    u32x4 a[P][2 * kAhead], b[NT][2 * kAhead];
#pragma unroll
    for (int i = 0; i < 2 * kAhead; ++i) {
      const int step = base + (i >> 1) * kStride + (i & 1);
      if (step < steps) {
#pragma unroll
        for (int p = 0; p < P; ++p) a[p][i] = chunk(from_w[p], step);
#pragma unroll
        for (int t = 0; t < NT; ++t) b[t][i] = chunk(from_x[t], step);
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) a[p][i] = u32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t) b[t][i] = u32x4{0, 0, 0, 0};
      }
    }
#pragma unroll
    for (int i = 0; i < 2 * kAhead; ++i)
#pragma unroll
      for (int p = 0; p < P; ++p)
#pragma unroll
        for (int t = 0; t < NT; ++t) acc[p][t] = mma16<T>(a[p][i], b[t][i], acc[p][t]);
  }
  if (steps * kStep < k && wave == WAVES - 1) {  // the rest of k, by elements
    const auto rest = [&](const char* row) {
      Pack<T, E> v;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int32_t c = steps * kStep + quarter * E + e;
        v.x[e] = c < k ? ((const M*)row)[c] : (M)0.f;
      }
      return __builtin_bit_cast(u32x4, v);
    };
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const u32x4 b = rest(from_x[t]);
#pragma unroll
      for (int p = 0; p < P; ++p) acc[p][t] = mma16<T>(rest(from_w[p]), b, acc[p][t]);
    }
  }
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4*>(&part[wave][p][t * 16 + r16][quarter * 4]) = acc[p][t];
  __syncthreads();
  if (threadIdx.x >= NT * 64) return;
  const int row = threadIdx.x >> 2, c = (threadIdx.x & 3) * 4;
  float v[P][4];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    f32x4 sum = *reinterpret_cast<const f32x4*>(&part[0][p][row][c]);
#pragma unroll 3
    for (int q = 1; q < WAVES; ++q) sum += *reinterpret_cast<const f32x4*>(&part[q][p][row][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[p][e] = sum[e];
  }
  typename Fin::template Lane<4> at;
  fin.begin(at, col0 + c);
  fin.put(at, row0 + row, v[0], v[P - 1]);
  if constexpr (Fin::kSums) fin.end(at, 4, (int64_t)blockIdx.y * NT + wave);
}
