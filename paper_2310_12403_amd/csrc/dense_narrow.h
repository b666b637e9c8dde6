// Dense layers of up to 128 by 128 in 16 bits, for any number of rows: bound by memory, and next to it by what an activation costs, so that
// nothing is moved that need not be.  Included by dense.hip.
//
// A wave takes 32 rows at a time and has them in its registers, as the matrix units' operands, straight from memory: a lane has 8 elements of
// its row for each 16 of k.  The weight lies in LDS for the whole of a block's life, fragment by fragment.  C's columns are in a lane's
// registers and its row is the lane's; after an exchange between the halves of the wave (swap_halves) a lane has 8 neighbouring columns, 16
// bytes, which is how residual, gradients and results are read and written, and what the next product takes as an operand.
#pragma once

// 16 bytes of a row of dim >= 8 columns from column `col` on, of rows of any alignment.  Where the row ends before them: the row's last 16, to be
// put right by mend_chunk when they have arrived.
template <int T>
__device__ __forceinline__ u32x4 load_chunk(const char* row, int col, int dim) {
  const int at = col < dim - 8 ? col : dim - 8;
  return __builtin_bit_cast(u32x4, Pack<T, 8>::load(row + at * 2));
}
// columns col .. col + 7 of what load_chunk has read, zeros behind column `dim` (16 * step: the first column of the lanes' chunks)
// EXACT, here and below: a row has as many columns as the kernel's tiles.
template <bool EXACT>
__device__ __forceinline__ u32x4 mend_chunk(u32x4 v, int step, int half, int dim) {
  if (EXACT || step * 16 + 16 <= dim) return v;
  const int lost = step * 16 + half * 8 - (dim - 8);  // columns that are not there
  if (lost <= 0) return v;
  if (lost >= 8) return u32x4{0, 0, 0, 0};
  typedef unsigned __int128 Bits;
  return __builtin_bit_cast(u32x4, __builtin_bit_cast(Bits, v) >> (16 * lost));
}
template <int T>
__device__ __forceinline__ void store_chunk(char* row, int step, int half, int dim, u32x4 v) {
  const int col = step * 16 + half * 8;
  char* const at = row + col * 2;
  if (step * 16 + 16 <= dim || col + 8 <= dim) {
    __builtin_bit_cast(Pack<T, 8>, v).store(at);
    return;
  }
  const int there = dim - col;
  if (there <= 0) return;
  int i = 0;
  if (there & 4) Pack<T, 4>(__builtin_bit_cast(Pack<T, 4>, u32x2{v[0], v[1]})).store(at), v[0] = v[2], v[1] = v[3], i = 4;
  if (there & 2) Pack<T, 2>(__builtin_bit_cast(Pack<T, 2>, v[0])).store(at + i * 2), v[0] = v[1], i += 2;
  if (there & 1) Pack<T, 1>(__builtin_bit_cast(Pack<T, 1>, (uint16_t)v[0])).store(at + i * 2);
}

// The rows of a wave's tile, chunk by chunk: 16 columns' two, one of them the lane's.  EXACT: at addresses of multiples of 16, and what lies behind
// the last row is neither read (zeros) nor written, without a branch: a wait for a load then counts exactly what was sent behind it.  Else a row
// behind the last one reads as the last one, and a tile as the last one.
template <int T, bool EXACT>
struct NarrowRows {
  char* base;  // the lane's row, or the tile's first
  int at, dim;
  bool live;
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ NarrowRows(const void* p, uint32_t tile, uint32_t tiles, int64_t n, int dim_, int lane) : dim(dim_) {
    const int64_t row = (int64_t)tile * 32;
    if constexpr (EXACT) {
      const int64_t left = n - row;
      base = (char*)p + row * dim * 2;
      rsrc = __builtin_amdgcn_make_buffer_rsrc(base, 0, left <= 0 ? 0 : (left < 32 ? (int)left : 32) * dim * 2, 0x00020000);
      at = (lane & 31) * dim * 2 + (lane >> 5) * 16;
    } else {
      const uint32_t t = tile < tiles ? tile : tiles - 1;
      const int64_t last = n - 1 - (int64_t)t * 32;
      const int r = lane & 31;
      live = row + r < n;
      base = (char*)p + (int64_t)t * 32 * dim * 2;
      at = (r < last ? r : (int)last) * dim * 2;
    }
  }
  __device__ __forceinline__ u32x4 load(int step, int half) const {
    if constexpr (EXACT) return __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + step * 32, 0, 0);
    else return load_chunk<T>(base + at, step * 16 + half * 8, dim);
  }
  __device__ __forceinline__ void store(int step, int half, u32x4 v) const {
    if constexpr (EXACT) __builtin_amdgcn_raw_buffer_store_b128(v, rsrc, at + step * 32, 0, 0);
    else if (live) store_chunk<T>(base + at, step, half, dim, v);
  }
};

// Columns 16 h + {0..3, 8..11} (lanes 0 to 31) and 16 h + {4..7, 12..15} (the others), packed, into 16 h + {0..7} and 16 h + {8..15}: what a
// tile's registers hold into 16 bytes of a row; and back, being its own reverse.
__device__ __forceinline__ u32x4 swap_halves(u32x4 v) {
  const auto a = __builtin_amdgcn_permlane32_swap(v[0], v[2], false, false), b = __builtin_amdgcn_permlane32_swap(v[1], v[3], false, false);
  return u32x4{a[0], b[0], a[1], b[1]};
}

struct NarrowLayer {
  const char *x, *w, *bias;
  int64_t n;
  int32_t k, m;
  float alpha, results;  // (of a gradient: what is multiplied into dz, and what into the results)
  int act;
};

// The weight's fragments in LDS, a kilobyte each, in a lane's order: [MT][KS] of W as the product with x takes it.  All threads of the block.
template <int T, int KS, int MT>
__device__ __forceinline__ void place_weight(const NarrowLayer& l, char* lds) {
  for (int i = threadIdx.x; i < MT * KS * 64; i += blockDim.x) {
    const int lane = i & 63, f = i >> 6, row = f / KS * 32 + (lane & 31), col = f % KS * 16 + (lane >> 5) * 8;
    *reinterpret_cast<u32x4*>(lds + i * 16) =
        row < l.m ? mend_chunk<false>(load_chunk<T>(l.w + (int64_t)row * l.k * 2, col, l.k), f % KS, lane >> 5, l.k) : u32x4{0, 0, 0, 0};
  }
}
template <int T, int MT>
__device__ __forceinline__ void place_bias(const NarrowLayer& l, float* lds) {
  for (int i = threadIdx.x; i < MT * 32; i += blockDim.x) lds[i] = l.bias != nullptr && i < l.m ? (float)((const typename Element<T>::M*)l.bias)[i] : 0.f;
}
__device__ __forceinline__ u32x4 fragment_at(const char* lds, int f) { return *reinterpret_cast<const u32x4*>(lds + f * 1024 + lane_id() * 16); }
// a tile's sums begin as the biases of its 32 columns
__device__ __forceinline__ f32x16 begin_with(const float* bias) {
  f32x16 z;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float f[4];
    load_elements<COOP_F32, 4>(bias + q * 8 + (lane_id() >> 5) * 4, f);
#pragma unroll
    for (int e = 0; e < 4; ++e) z[4 * q + e] = f[e];
  }
  return z;
}

template <int T>
__device__ __forceinline__ u32x4 pack8(const float (&f)[8]) {
  Pack<T, 8> x;
  x.set(f);
  return __builtin_bit_cast(u32x4, x);
}
template <int T>
__device__ __forceinline__ void unpack8(u32x4 v, float (&f)[8]) {
  __builtin_bit_cast(Pack<T, 8>, v).get(f);
}

constexpr int kNarrowForwardWaves = 4;
template <int T, int KS, int MT, bool EXACT>
__global__ __launch_bounds__(kNarrowForwardWaves* kWave) void k_narrow(NarrowLayer l, const char* __restrict__ residual, char* __restrict__ out,
                                                                       float* __restrict__ pre, uint32_t tiles) {
  __shared__ __attribute__((aligned(16))) char lds[MT * KS * 1024];
  __shared__ __attribute__((aligned(16))) float bias[MT * 32];
  place_weight<T, KS, MT>(l, lds);
  place_bias<T, MT>(l, bias);
  __syncthreads();
  const int lane = lane_id(), half = lane >> 5;
  const uint32_t step = gridDim.x * kNarrowForwardWaves;
  uint32_t tile = blockIdx.x * kNarrowForwardWaves + uniform_wave_in_block();
  if (tile >= tiles) return;
  u32x4 xf[KS], res[2 * MT];
  const auto load_x = [&](uint32_t to) {
    const NarrowRows<T, EXACT> r(l.x, to, tiles, l.n, l.k, lane);
#pragma unroll
    for (int s = 0; s < KS; ++s) xf[s] = r.load(s, half);
  };
  load_x(tile);
  if (residual != nullptr) {
    const NarrowRows<T, EXACT> r(residual, tile, tiles, l.n, l.m, lane);
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) res[i] = r.load(i, half);
  }
  for (; tile < tiles; tile += step) {
    const int64_t row = (int64_t)tile * 32 + (lane & 31);
    const bool live = row < l.n;
    f32x16 z[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) z[i] = begin_with(bias + i * 32);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const u32x4 x = mend_chunk<EXACT>(xf[s], s, half, l.k);
#pragma unroll
      for (int i = 0; i < MT; ++i) z[i] = mma<T>(fragment_at(lds, i * KS + s), x, z[i]);
      if (s & 1) __builtin_amdgcn_sched_barrier(0);
    }
    load_x(tile + step);
    const NarrowRows<T, EXACT> next(residual, tile + step, tiles, l.n, l.m, lane), to(out, tile, tiles, l.n, l.m, lane);
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = 2 * i + h;
        float v[8], r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = z[i][8 * h + e];
        if (pre != nullptr && live) {
          const float a[4] = {v[0], v[1], v[2], v[3]}, b[4] = {v[4], v[5], v[6], v[7]};
          store_columns<COOP_F32, 4>(pre + row * l.m, c * 16 + half * 4, l.m, a);
          store_columns<COOP_F32, 4>(pre + row * l.m, c * 16 + 8 + half * 4, l.m, b);
        }
        act_values(v, l.act);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= l.alpha;
        if (residual != nullptr) {
          unpack8<T>(swap_halves(mend_chunk<EXACT>(res[c], c, half, l.m)), r);
          res[c] = next.load(c, half);
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += r[e];
        }
        to.store(c, half, swap_halves(pack8<T>(v)));
        __builtin_amdgcn_sched_barrier(0);  // (or the compiler spreads the chunks' work over more registers than there are)
      }
  }
}

// The whole gradient in one pass over x and dout: z once more, dz, dx, and the sums for the weight's gradient and the bias's.  A block has 32 rows
// for each of its eight waves at a time, two to a SIMD, so that one's activations (some 130 cycles a value of gelu's slope: as much as the memory takes)
// run beside the other's products.  dW is dealt to the waves by tiles of 32 x 32 (of few tiles, by parts of the rows too): the rows of x and dz of all of
// them meet in LDS, where the product over the rows reads them transposed; so is the weight, which is there once, for dx.  (REST: what dz loses to its type lies
// beside it there, and is multiplied too.)
template <int T, int KS, int MT, bool REST = false>
struct NarrowBackward {
  static constexpr int kWaves = 8, KT = KS / 2, kTiles = KT * MT;
  static constexpr int kMine = kTiles > kWaves ? kTiles / kWaves : 1;     // tiles of dW that a wave has, neighbours along m
  static constexpr int kShares = kTiles < kWaves ? kWaves / kTiles : 1;   // waves that share a tile, by their rows
  typedef Staged<T, MT * 32, true, kNarrow, 1> Z;
  typedef Staged<T, KT * 32, true, kNarrow, 1> X;
  static constexpr int kZ = (REST ? 2 : 1) * Z::kBytes, kOwn = kZ + X::kBytes, kWeight = MT * KS * 1024, kLds = kWeight + kWaves * kOwn;
  static_assert(kLds <= 160 * 1024 && kWaves * MT * 32 * 4 <= kLds - kWeight, "a CU's LDS");
};
constexpr int kNarrowSums = 8;  // columns behind those of dW in a part: the bias's gradient in the first of them

// the waves' LDS is written, or read, by all of them (loads from memory stay under way)
__device__ __forceinline__ void narrow_meet() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// The same number, of which the compiler does not know it: what follows from it is computed anew, rather than kept in registers that are needed.
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// parts: [blocks][kShares][m][width], of the `width - kNarrowSums` columns of dW (none: it is not asked for) and db's; null: neither is.
template <int T, int KS, int MT, bool EXACT, bool REST>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_narrow_grad(NarrowLayer l, const char* __restrict__ dout, char* __restrict__ dx,
                                                                                                float* __restrict__ parts, int32_t width, uint32_t tiles) {
  typedef NarrowBackward<T, KS, MT, REST> B;
  typedef typename Element<T>::M M;
  constexpr int KT = B::KT, kOwn = B::kOwn;
  extern __shared__ char lds[];
  const int wave = uniform_wave_in_block(), lane = lane_id(), half = lane >> 5, r32 = lane & 31;
  char* const staged = lds + B::kWeight;  // of each wave: dz, what it lost, then x
  char* const own_z = staged + wave * kOwn;
  char* const own_x = own_z + B::kZ;
  // the weight, row by row, as the product over its rows reads it
  for (int i = threadIdx.x; i < MT * 32 * KS * 2; i += 512) {
    const int row = i / (KS * 2), chunk = i % (KS * 2);
    *reinterpret_cast<u32x4*>(lds + row * (KS * 32) + ((chunk ^ B::X::swizzle(row)) << 4)) =
        row < l.m ? mend_chunk<false>(load_chunk<T>(l.w + (int64_t)row * l.k * 2, chunk * 8, l.k), chunk >> 1, chunk & 1, l.k) : u32x4{0, 0, 0, 0};
  }
  // biases as a product's operand: times a column of ones
  uint32_t bias[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int c = i * 32 + r32;
    const M b = l.bias != nullptr && half == 0 && c < l.m ? ((const M*)l.bias)[c] : (M)0.f;
    bias[i] = __builtin_bit_cast(uint16_t, b);
  }
  const uint32_t one = half == 0 ? __builtin_bit_cast(uint16_t, (M)1.f) : 0;
  const bool want_dw = width > kNarrowSums;
  const int mine = wave / B::kShares * B::kMine, mine_t = mine / MT, mine_i = mine % MT, share = wave % B::kShares;
  f32x16 dw[B::kMine];
#pragma unroll
  for (int i = 0; i < B::kMine; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) dw[i][e] = 0.f;
  float db[MT][2][4];  // of two rows' sums each: lanes whose fifth bit is set have the columns 8 further on
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) db[i][0][e] = db[i][1][e] = 0.f;
  u32x4 xf[KS], dy[2 * MT];
  const auto load_x = [&](uint32_t to) {
    const int lane = anew(lane_id());
    const NarrowRows<T, EXACT> r(l.x, to, tiles, l.n, l.k, lane);
#pragma unroll
    for (int s = 0; s < KS; ++s) xf[s] = r.load(s, lane >> 5);
  };
  const auto load_dy = [&](uint32_t to) {
    const int lane = anew(lane_id());
    const NarrowRows<T, EXACT> r(dout, to, tiles, l.n, l.m, lane);
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) dy[i] = r.load(i, lane >> 5);
  };
  // (a wave whose tile there is not goes along with zeros: the block's waves meet)
  uint32_t first = blockIdx.x * B::kWaves;
  load_x(first + wave);
  load_dy(first + wave);
  narrow_meet();
  for (; first < tiles; first += gridDim.x * B::kWaves) {
    const uint32_t next = first + gridDim.x * B::kWaves + wave;
    const int64_t row = (int64_t)(first + wave) * 32 + r32;
    const bool live = row < l.n, whole = (int64_t)(first + wave) * 32 + 32 <= l.n;
    u32x4 dz[2 * MT];
    const int r = anew(r32);
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      xf[s] = mend_chunk<EXACT>(xf[s], s, anew(lane) >> 5, l.k);
      if (!EXACT && !whole && !live) xf[s] = u32x4{0, 0, 0, 0};
    }
#pragma unroll
    for (int s = 0; s < KS; ++s)
      *reinterpret_cast<u32x4*>(own_x + r * (KT * 64) + (((2 * s + half) ^ B::X::swizzle(r)) << 4)) = xf[s];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      f32x16 z;
      if (l.act != COOP_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 16; ++e) z[e] = 0.f;
        z = mma<T>(u32x4{(uint32_t)anew((int)bias[i]), 0, 0, 0}, u32x4{(uint32_t)anew((int)one), 0, 0, 0}, z);
        const int m = i * 32 + r;
#pragma unroll
        for (int s = 0; s < KS; ++s)
          z = mma<T>(*reinterpret_cast<const u32x4*>(lds + m * (KS * 32) + (((2 * s + half) ^ B::X::swizzle(m)) << 4)), xf[s], z);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = 2 * i + h;
        dz[c] = mend_chunk<EXACT>(dy[c], c, anew(lane) >> 5, l.m);
        if (!EXACT && !whole && !live) dz[c] = u32x4{0, 0, 0, 0};
        float d[8];
        unpack8<T>(swap_halves(dz[c]), d);
        if (l.act != COOP_ACT_NONE) {
          float s[8], value[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] = z[8 * h + e];
          act_slopes(s, value, l.act);
#pragma unroll
          for (int e = 0; e < 8; ++e) d[e] = whole || live ? d[e] * l.alpha * s[e] : 0.f;
          dz[c] = swap_halves(pack8<T>(d));
          if constexpr (REST) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s[e] = lost_to<T>(d[e]);
            *reinterpret_cast<u32x4*>(own_z + B::Z::kBytes + r * (MT * 64) + (((2 * c + half) ^ B::Z::swizzle(r)) << 4)) = swap_halves(pack8<T>(s));
          }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(d[e]), __float_as_uint(d[e + 4]), false, false);
          db[i][h][e] += __uint_as_float(both[0]) + __uint_as_float(both[1]);
        }
        *reinterpret_cast<u32x4*>(own_z + r * (MT * 64) + (((2 * c + half) ^ B::Z::swizzle(r)) << 4)) = dz[c];
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    load_x(next);
    if (dx != nullptr) {
      const int at = anew(lane);
      const NarrowRows<T, EXACT> to(dx, first + wave, tiles, l.n, l.k, at);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        f32x16 v;
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = 0.f;
#pragma unroll
        for (int s = 0; s < 2 * MT; ++s) {
          const u32x4 w = B::X::fragment(lds, t * 32, s, at);
          v = mma<T>(w, dz[s], v);
          if constexpr (REST) {  // (what the lane has written)
            const int row = at & 31;
            v = mma<T>(w, *reinterpret_cast<const u32x4*>(own_z + B::Z::kBytes + row * (MT * 64) + (((2 * s + (at >> 5)) ^ B::Z::swizzle(row)) << 4)), v);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          float f[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] = v[8 * h + e] * l.results;
          to.store(2 * t + h, at >> 5, swap_halves(pack8<T>(f)));
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    load_dy(next);  // (not before: what is on its way takes registers)
    if (want_dw) {
      narrow_meet();
      const int at = anew(lane);
      for (int w = share; w < B::kWaves; w += B::kShares) {
        const char* z = staged + w * kOwn;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const u32x4 a = B::X::fragment(z + B::kZ, mine_t * 32, kk, at);
#pragma unroll
          for (int i = 0; i < B::kMine; ++i) {
            dw[i] = mma<T>(a, B::Z::fragment(z, (mine_i + i) * 32, kk, at), dw[i]);
            if constexpr (REST) dw[i] = mma<T>(a, B::Z::fragment(z + B::Z::kBytes, (mine_i + i) * 32, kk, at), dw[i]);
          }
        }
      }
      narrow_meet();
    }
  }
  if (parts == nullptr) return;
  // (the staged rows are read: the waves meet behind their last reads, or have read none)
  float* const sums = reinterpret_cast<float*>(staged);
  narrow_meet();
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float v = db[i][h][e];
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) v += __shfl_xor(v, off, kWave);
        if ((lane & 15) == 0) sums[wave * (MT * 32) + i * 32 + h * 16 + (lane >> 4 & 1) * 8 + half * 4 + e] = v;
      }
  narrow_meet();
  float* const to = parts + ((int64_t)blockIdx.x * B::kShares + share) * l.m * width;
  if (want_dw) {
#pragma unroll
    for (int i = 0; i < B::kMine; ++i) {
      const int m = (mine_i + i) * 32 + r32;
      if (m >= l.m) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int col = mine_t * 32 + q * 8 + half * 4;
        const float f[4] = {dw[i][4 * q], dw[i][4 * q + 1], dw[i][4 * q + 2], dw[i][4 * q + 3]};
        if (col < width - kNarrowSums) store_elements<COOP_F32, 4>(to + (int64_t)m * width + col, f);
      }
    }
  }
  // (the shares' parts are added up, so that the first has the block's and the others zeros)
  for (int i = threadIdx.x; i < B::kShares * l.m; i += 512) {
    const int part = i / l.m, m = i - part * l.m;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (part == 0)
      for (int w = 0; w < B::kWaves; ++w) v[0] += sums[w * (MT * 32) + m];
    v[0] *= l.results;
    store_elements<COOP_F32, 4>(parts + (((int64_t)blockIdx.x * B::kShares + part) * l.m + m) * width + width - kNarrowSums, v);
  }
}
