// The gradient of a dense layer that is small altogether, where launches cost more than products: one kernel makes dz (or none, where it is dout),
// and one has the input's gradient, the weight's and the bias's in blocks of their own.  Included by dense.hip.
//
// As in dense_few.h a block has 16 columns by 32 rows of a result and its waves deal the common dimension among themselves.  An operand that
// has that dimension as its row number comes 16 bytes of a row at a time, 16 columns of a step, and is turned in the wave's own LDS.
//
// With REST dz is the sum of two numbers of the operands' type and multiplied by both.  (All of them so: 3,001 x 100 x 275 gated both ways 55 us for 39, 1,024 x
// 256 x 256 14.1 for 11.0.)
#pragma once

struct SmallGrad {
  const char *dz, *x, *w, *w2;
  int64_t n, ld, second, rest;  // dz: bytes of a row, elements from a pair's first part to its second, bytes to its rest
  int32_t k, m;
  uint32_t dx_blocks, dw_blocks, k_tiles;  // (and behind them 64 columns of the bias's gradient a block)
  const float *part, *part2;
  int64_t part_rows;
  float *db, *db2;
};

// kSmallLength: bytes of the common dimension, 12 steps for each wave: longer ones take too long in the few blocks of a weight's gradient.  (Against tiles, 16 bits: 100 x
// 275 gated, 3,000 rows 30.0 us for 37.5, 3,700 34.9 for 39.2, with what was kept 41.5 for 40.5; 64 x 200 3,000 18.9 for 26.6, 4,500 26.2 both, 5,500 30.3 for 26.6.
// fp32, 100 x 100 gated, 1,500 rows 21.4 for 34.2, 2,300 27.7 for 34.0, 3,000 36.0 for 35.7.  Against dense_narrow.h it ends earlier: 64 x 64, 1,500 rows 15.0 for
// 16.5, 2,200 17.8 for 15.6, 3,000 20.4 for 15.5.)  8 waves for 16, which are idle where it is short: bf16 1,024 x 256 x 256 11.0 us for 13.1,
// 256 x 1,024 x 512 13.1 for 19.9; 4: 12.5 and 12.5, and 31.5 for 26.4 with 3,001 rows.
constexpr int kSmallWaves = 8, kSmallRows = 32, kSmallLength = 12 * 8 * 64;

// 16 bytes of a row from column `col` on, zeros behind column `dim`
template <int T>
__device__ __forceinline__ u32x4 load_some(const char* row, int64_t col, int64_t dim) {
  typedef typename Element<T>::M M;
  constexpr int E = kE<T>;
  if (col + E <= dim) return __builtin_bit_cast(u32x4, Pack<T, E>::load((const M*)row + col));
  Pack<T, E> v;
#pragma unroll
  for (int e = 0; e < E; ++e) v.x[e] = col + e < dim ? ((const M*)row)[col + e] : (M)0.f;
  return __builtin_bit_cast(u32x4, v);
}

// What a lane loads of a step of an operand whose rows are the common dimension, and the fragment that it is (lds: the wave's kilobyte).
template <int T>
__device__ __forceinline__ u32x4 load_strided(const char* base, int64_t ld, int64_t row0, int64_t rows, int64_t col0, int64_t dim) {
  constexpr int E = kE<T>, kEach = 16 / E;  // lanes of a row
  const int64_t r = row0 + lane_id() / kEach;
  return r < rows ? load_some<T>(base + r * ld, col0 + lane_id() % kEach * E, dim) : u32x4{0, 0, 0, 0};
}
template <int T>
__device__ __forceinline__ u32x4 turned(char* lds, u32x4 v) {
  const int lane = lane_id(), t = lane & 15, quarter = lane >> 4;
  asm volatile("" ::: "memory");  // (a wave's reads and writes of LDS are done in their order)
  *reinterpret_cast<u32x4*>(lds + lane * 16) = v;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  u32x4 f;
  if constexpr (T == COOP_F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const uint32_t*>(lds + (quarter * 4 + j) * 64 + t * 4);
  } else {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const char* at = lds + (quarter * 8 + q * 4 + (t >> 2)) * 32 + (t & 3) * 8;
      const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(LdsByte*)at));
      f[2 * q] = y[0];
      f[2 * q + 1] = y[1];
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  return f;
}

template <int T, bool PAIR, bool REST>
__global__ __launch_bounds__(kSmallWaves* kWave) void k_small_grad(SmallGrad g, Gradient to_x, Gradient to_w) {
  constexpr int E = kE<T>, kStep = 4 * E, kAhead = 2, Z = REST ? 4 : 2;  // Z: fragments of dz
  __shared__ __attribute__((aligned(16))) char lds[kSmallWaves * 3 * 1024];
  static_assert(kSmallWaves * kSmallRows * 16 * 4 <= (int)sizeof(lds), "the sums lie where the fragments did");
  const int wave = uniform_wave_in_block(), lane = lane_id(), r16 = lane & 15, quarter = lane >> 4;
  char* const own = lds + wave * 3 * 1024;
  uint32_t block = blockIdx.x;
  if (block >= g.dx_blocks + g.dw_blocks) {  // the bias's gradient: the waves deal the parts' rows
    block -= g.dx_blocks + g.dw_blocks;
    const uint32_t each = (uint32_t)((g.m + kWave - 1) / kWave);
    const bool second = block >= each;
    const float* part = second ? g.part2 : g.part;
    const int32_t c = (int32_t)(second ? block - each : block) * kWave + lane;
    float(*const sums)[kWave] = reinterpret_cast<float(*)[kWave]>(lds);
    float sum = 0.f;
    if (c < g.m) {
#pragma unroll 8
      for (int64_t r = wave; r < g.part_rows; r += kSmallWaves) sum += part[r * g.m + c];
    }
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave != 0 || c >= g.m) return;
    sum = 0.f;
#pragma unroll
    for (int w = 0; w < kSmallWaves; ++w) sum += sums[w][lane];
    (second ? g.db2 : g.db)[c] = sum;
    return;
  }
  const bool of_x = block >= g.dw_blocks;  // (the weight's first: they take longer)
  if (of_x) block -= g.dw_blocks;
  const int64_t col0 = (int64_t)(block % g.k_tiles) * 16, row0 = (int64_t)(block / g.k_tiles) * kSmallRows, ldk = (int64_t)g.k * kElem<T>;
  f32x4 acc[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
  if (of_x) {  // dz by its rows, the weight turned
    const char* rows[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t r = row0 + t * 16 + r16;
      rows[t] = g.dz + (r < g.n ? r : g.n - 1) * g.ld;  // (what is not there: the last one's, and nothing is stored)
    }
    const int steps = (g.m + kStep - 1) / kStep, all = PAIR ? 2 * steps : steps;
    for (int first = wave; first < all; first += kSmallWaves * kAhead) {
      u32x4 a[kAhead], b[kAhead][Z];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        int s = first + i * kSmallWaves;
        const bool there = s < all, other = PAIR && s >= steps;
        if (other) s -= steps;
        a[i] = there ? load_strided<T>(other ? g.w2 : g.w, ldk, (int64_t)s * kStep, g.m, col0, g.k) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < Z; ++t)
          b[i][t] = there ? load_some<T>(rows[t & 1] + (other ? g.second * kElem<T> : 0) + (t & 2 ? g.rest : 0), (int64_t)s * kStep + quarter * E, g.m)
                          : u32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const u32x4 f = turned<T>(own, a[i]);
#pragma unroll
        for (int t = 0; t < Z; ++t) acc[t & 1] = mma16<T>(f, b[i][t], acc[t & 1]);
      }
    }
  } else {  // x and dz turned
    const int64_t steps = (g.n + kStep - 1) / kStep, cols = PAIR ? g.second + g.m : g.m;
    for (int64_t first = wave; first < steps; first += kSmallWaves * kAhead) {
      u32x4 a[kAhead], b[kAhead][Z];
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const int64_t s = first + i * kSmallWaves;  // (behind the last one: rows that are not there)
        a[i] = load_strided<T>(g.x, ldk, s * kStep, g.n, col0, g.k);
#pragma unroll
        for (int t = 0; t < Z; ++t) b[i][t] = load_strided<T>(g.dz + (t & 2 ? g.rest : 0), g.ld, s * kStep, g.n, row0 + (t & 1) * 16, cols);
      }
#pragma unroll
      for (int i = 0; i < kAhead; ++i) {
        const u32x4 f = turned<T>(own, a[i]);
#pragma unroll
        for (int t = 0; t < Z; ++t) acc[t & 1] = mma16<T>(f, turned<T>(own + (1 + (t & 1)) * 1024, b[i][t]), acc[t & 1]);
      }
    }
  }
  __syncthreads();
  float(*const sums)[kSmallRows][16] = reinterpret_cast<float(*)[kSmallRows][16]>(lds);
#pragma unroll
  for (int t = 0; t < 2; ++t) *reinterpret_cast<f32x4*>(&sums[wave][t * 16 + r16][quarter * 4]) = acc[t];
  __syncthreads();
  if (threadIdx.x >= kSmallRows * 4) return;
  const int row = threadIdx.x >> 2, c = (threadIdx.x & 3) * 4;
  f32x4 sum = *reinterpret_cast<const f32x4*>(&sums[0][row][c]);
#pragma unroll 3
  for (int q = 1; q < kSmallWaves; ++q) sum += *reinterpret_cast<const f32x4*>(&sums[q][row][c]);
  float v[4] = {sum[0], sum[1], sum[2], sum[3]}, none[4] = {0.f, 0.f, 0.f, 0.f};
  const Gradient& fin = of_x ? to_x : to_w;
  typename Gradient::Lane<4> at;
  fin.begin(at, (int32_t)col0 + c);
  fin.put(at, row0 + row, v, none);
}
