// Dense layers of up to 32 rows, one token first of all: bound by the weight, which is read once and straight into the matrix units' registers.
// Included by dense.hip.
//
// A block has 16 columns of the result, so that there are blocks for every CU, and all of k: its 16 waves deal it among themselves, 128 bytes of
// a row at a time, and their sums meet in LDS.  One launch; with k dealt to blocks in its place a second one that joins them (4,096 x 4,096 in
// bf16, one row: 13.2 us on the GPU, 14.8 a call).
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

constexpr int kFewRows = 32, kFewWaves = 16;

// NT: tiles of 16 rows of x
template <int T, int NT, bool PAIR>
__global__ __launch_bounds__(kFewWaves* kWave) void k_few(const char* __restrict__ x, const char* __restrict__ w, const char* __restrict__ w2, int32_t n, int32_t k,
                                                           Forward<T, PAIR> fin) {
  typedef typename Element<T>::M M;
  constexpr int E = kE<T>, P = PAIR ? 2 : 1, kStep = 4 * E, kAhead = 2;  // elements of k in a step; pairs of steps on their way at a time
  __shared__ __attribute__((aligned(16))) float part[kFewWaves][P][NT * 16][16];
  const int wave = uniform_wave_in_block(), lane = lane_id(), r16 = lane & 15, quarter = lane >> 4;
  const int32_t col0 = (int32_t)blockIdx.x * 16;
  const int32_t col = col0 + r16 < fin.cols ? col0 + r16 : fin.cols - 1;  // (what is not there: the last one's, and nothing is stored)
  const int64_t ld = (int64_t)k * kElem<T>;
  const char* const from_w[2] = {w + col * ld, PAIR ? w2 + col * ld : nullptr};
  const char* from_x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) from_x[t] = x + (t * 16 + r16 < n ? t * 16 + r16 : n - 1) * ld;
  f32x4 acc[P][NT];
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[p][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = k / kStep;  // whole ones
  const auto chunk = [&](const char* row, int step) { return __builtin_bit_cast(u32x4, Pack<T, E>::load(row + (int64_t)step * 64 + quarter * 16)); };
  constexpr int kStride = kFewWaves * 2;
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
  if (steps * kStep < k && wave == kFewWaves - 1) {  // the rest of k, by elements
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
#pragma unroll 5
    for (int q = 1; q < kFewWaves; ++q) sum += *reinterpret_cast<const f32x4*>(&part[q][p][row][c]);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[p][e] = sum[e];
  }
  typename Forward<T, PAIR>::template Lane<4> at;
  fin.begin(at, col0 + c);
  fin.put(at, row, v[0], v[P - 1]);
}
