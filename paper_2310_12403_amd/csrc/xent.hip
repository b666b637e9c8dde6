// Softmax cross entropy over a large vocabulary without the logits kept, and its gradient.
//
// With z = alpha H W^T (H [n, dim] hidden states, W [vocab, dim]), t the rows' targets:
//   lse_i = log sum_v exp z_iv,   loss_i = lse_i - z_i,t(i),
//   G_iv = alpha dloss_i (exp(z_iv - lse_i) - [v = t(i)]),   dH = G W,   dW = G^T H.
// Forward: one product, whose tiles stay in registers and leave as a running maximum and sum per row.  Backward: the logits again, a
// piece of the vocabulary at a time, left as G of that piece in 16 bits (32 for fp32), and the two products with it.
//
// The products run on the matrix units from tiles in LDS.  All three are the same kernel: C = A B^T over a common dimension k, where an
// operand either has k as its contiguous dimension (rows of 128 bytes of k per stage) or as its row number (then its fragments are
// transposed on the way from LDS to the registers).  The columns of C lie on the lanes and its rows in a lane's registers, so C is
// computed as vocabulary x hidden for the logits: a lane then holds many logits of one row of H, and neither maximum, sum nor target
// takes another lane until the end.
#include <type_traits>

#include "coop_internal.h"
#include "elements.h"

namespace coop {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char LdsByte;

constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.693147180559945309f;
// Bytes of k per row and stage: 64 (32 elements of 16 bits, 16 of 32), four stages in LDS, or 128, two of them.  One is read, the others
// are on their way.  Rows of 64 bytes are half a cache line, so operands with k contiguous take 128.
constexpr int kWide = 128, kNarrow = 64;
constexpr float kNoMax = -3.402823466e38f;

template <int T> constexpr int kElem = T == COOP_F32 ? 4 : 2;

// One 16-byte fragment of each operand into a 32 x 32 tile of C: 16 of k in 16 bits, 8 in 32.
template <int T>
__device__ __forceinline__ f32x16 mma(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (T == COOP_F16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  } else if constexpr (T == COOP_BF16) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
    return c;
  }
}

// An operand in memory: rows of `ld` bytes (a multiple of 16, as is the base).  k contiguous: `rows` rows, `k` bytes of each are there.
// k strided: `k` rows (one for each k), `rows` bytes of each are there.
struct Operand {
  const char* base;
  int64_t ld, rows, k;
};

// How a stage of R rows of an operand lies in LDS, in 16-byte slots filled in order by the loads, 64 to a wave's load.
//   k contiguous: a row's 4 or 8 chunks, exchanged by the row's number so that what 8 or 16 lanes read together lies in different banks;
//   k strided: a row of k holds R elements; its chunks are exchanged by k so that what one fragment reads lies in different banks.
// Both exchanges are an exclusive or with bits that neither the next tile of 32 rows nor the next step of k changes.
template <int T, int R, bool STRIDED, int SIZE, int WAVES>
struct Staged {
  static constexpr int kBytes = R * SIZE, kK = SIZE / kElem<T>;
  static constexpr int kChunks = STRIDED ? R * kElem<T> / 16 : SIZE / 16;  // of a row
  static constexpr int kAll = kBytes / 1024;                                      // loads of a stage
  static_assert(kAll % WAVES == 0 || kAll < WAVES, "loads are dealt to the waves evenly, or the first ones have one");
  static constexpr int kLoads = kAll / WAVES;  // that every wave has
  static __device__ __forceinline__ int swizzle(int row) {
    if constexpr (!STRIDED) return SIZE == 128 ? (row & 7) ^ (row >> 3 & 1) : (row >> 1 & 3) ^ (row >> 3 & 1);
    else if constexpr (T == COOP_F32) return (row >> 2 & 1) << 3 & (kChunks - 1);
    else return (((row & 3) | (row >> 3 & 1) << 2) << 2) & (kChunks - 1);
  }
  // A stage that is to be loaded: where it begins in memory, how many of the memory layout's rows there are, and bytes in each.
  struct Place {
    const char* p;
    int there, in_row;
    __device__ __forceinline__ Place() {}
    __device__ __forceinline__ Place(const Operand& op, int64_t row0, int64_t k0) {
      const int64_t most = 0x7FFFFFFF, rows = STRIDED ? op.k - k0 : op.rows - row0, bytes = STRIDED ? op.rows - row0 * kElem<T> : op.k - k0 * kElem<T>;
      p = op.base + (STRIDED ? k0 * op.ld + row0 * kElem<T> : row0 * op.ld + k0 * kElem<T>);
      there = (int)(rows < 0 ? 0 : rows < most ? rows : most);
      in_row = (int)(bytes < 0 ? 0 : bytes < most ? bytes : most);
    }
    __device__ __forceinline__ void next(int ld) {
      if constexpr (STRIDED) p += (int64_t)ld * kK, there -= kK;
      else p += SIZE, in_row -= SIZE;
    }
  };
  // What a lane loads of every stage: offsets from the stage's beginning.  What is not there reads as zero: rows because they lie behind
  // the last record; chunks behind a row's end because their offsets are put there, with k strided once and for all.
  struct Loads {
    static constexpr int kMine = (kAll + WAVES - 1) / WAVES, kNowhere = 0x3FFFFFFF;
    int ld, chunk, at[kMine];
    __device__ __forceinline__ void begin(const Operand& op, const Place& first) {
      const int wave = uniform_wave_in_block(), lane = lane_id();
      ld = (int)op.ld;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int slot = (i * WAVES + wave) * kWave + lane, row = slot / kChunks;
        chunk = ((slot % kChunks) ^ swizzle(row)) * 16;  // (k contiguous: the same for all of a lane's loads)
        at[i] = row * ld + chunk;
        if (STRIDED && chunk >= first.in_row) at[i] = kNowhere;
      }
    }
    // what the loads of a stage have in common
    struct Stage {
      __amdgpu_buffer_rsrc_t rsrc;
      int off;
    };
    __device__ __forceinline__ Stage stage(const Place& s) const {
      constexpr int kRows = STRIDED ? kK : R;
      const int rows = s.there < kRows ? s.there : kRows, in_row = s.in_row < ld ? s.in_row : ld, last = (rows - 1) * ld + in_row;
      const int records = (rows < in_row ? rows : in_row) > 0 ? last : 0;
      return Stage{__builtin_amdgcn_make_buffer_rsrc((void*)s.p, 0, records, 0x00020000), !STRIDED && chunk >= s.in_row ? kNowhere : 0};
    }
    __device__ __forceinline__ void start(const Stage& s, char* lds, int i) const {
      const int l = i * WAVES + uniform_wave_in_block();
      if (kAll < WAVES && l >= kAll) return;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(s.rsrc, (__attribute__((address_space(3))) void*)(LdsByte*)(lds + l * 1024), 16,
                                               STRIDED ? at[i] : at[i] + s.off, 0, 0, 0);
    }
  };
  // the fragment of rows row .. row + 31 at step kk of the stage
  static __device__ __forceinline__ u32x4 fragment(const char* lds, int row, int kk) {
    const int lane = lane_id();
    if constexpr (!STRIDED) {
      const int r = row + (lane & 31), chunk = kk * 2 + (lane >> 5);
      return *reinterpret_cast<const u32x4*>(lds + r * SIZE + ((chunk ^ swizzle(r)) << 4));
    } else if constexpr (T == COOP_F32) {
      const int m = row + (lane & 31);
      u32x4 f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = kk * 8 + (lane >> 5) * 4 + j;
        f[j] = *reinterpret_cast<const uint32_t*>(lds + k * (R * 4) + (((m >> 2) ^ swizzle(k)) << 4) + (m & 3) * 4);
      }
      return f;
    } else {
      // 16 lanes read 4 rows of k by 16 elements and get an element's 4 k each
      const int b = lane >> 4, t = lane & 15;
      u32x4 f;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int k = kk * 16 + (b >> 1) * 8 + q * 4 + (t >> 2), m = row + (b & 1) * 16 + (t & 3) * 4;
        const char* at = lds + k * (R * 2) + (((m >> 3) ^ swizzle(k)) << 4) + (m & 7) * 2;
        const i16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(LdsByte*)at);
        const u32x2 y = __builtin_bit_cast(u32x2, x);
        f[2 * q] = y[0];
        f[2 * q + 1] = y[1];
      }
      return f;
    }
  }
};

// A block's tile of C: WA x WB waves with TA x TB tiles of 32 x 32 each, rows of A by rows of B.  The stages of all of a block's tiles
// are one stream: while one is multiplied the next kStages - 1 are on their way, the first of the next tile among them.
template <int T, int WA, int WB, int TA, int TB, bool SA, bool SB, int SIZE>
struct Product {
  static constexpr int kWaves = WA * WB, kThreads = kWaves * kWave;
  static constexpr int kRowsA = WA * TA * 32, kRowsB = WB * TB * 32;
  static constexpr int kK = SIZE / kElem<T>, kSteps = SIZE / 32, kStages = 256 / SIZE;
  typedef Staged<T, kRowsA, SA, SIZE, kWaves> A;
  typedef Staged<T, kRowsB, SB, SIZE, kWaves> B;
  static constexpr int kStage = A::kBytes + B::kBytes, kLds = kStages * kStage;
  f32x16 acc[TA][TB];
  u32x4 fa[TA], fb[TB];  // the last step of the last stage that was read
  typename A::Loads loads_a;
  typename B::Loads loads_b;
  typename A::Place a, next_a;  // the stage that is loaded next, and the first one of the tile behind its
  typename B::Place b, next_b;
  typename A::Loads::Stage sa;
  typename B::Loads::Stage sb;
  int left;                     // stages of its tile that are to be loaded
  int slot;                     // where in LDS it goes; the one behind it is read next
  int stages;
  int step_rows;                // from tile to tile, of A; 0: there is one tile
  int64_t step_bytes;
  char* lds;

  __device__ __forceinline__ static int a0() { return uniform_wave_in_block() / WB * (TA * 32); }
  __device__ __forceinline__ static int b0() { return uniform_wave_in_block() % WB * (TB * 32); }
  // C's element j of a 32 x 32 tile: its row is the lane's own plus one that all lanes have; its column is lane & 31
  __device__ __forceinline__ static int own_row() { return (lane_id() >> 5) * 4; }
  __device__ __forceinline__ static constexpr int row_of(int j) { return (j >> 2) * 8 + (j & 3); }

  // to the next stage of the stream
  __device__ __forceinline__ void next() {
    a.next(loads_a.ld);
    b.next(loads_b.ld);
    --left;
    const bool done = left == 0;  // (chosen, not branched around: the products go on meanwhile)
    left = done ? stages : left;
    a.p = done ? next_a.p : a.p;
    a.there = done ? next_a.there : a.there;
    a.in_row = done ? next_a.in_row : a.in_row;
    b.p = done ? next_b.p : b.p;
    b.there = done ? next_b.there : b.there;
    b.in_row = done ? next_b.in_row : b.in_row;
    next_a.p += done ? step_bytes : 0;
    next_a.there -= done ? step_rows : 0;
    sa = loads_a.stage(a);
    sb = loads_b.stage(b);
  }
  // Of this wave's loads, those of the stage that is read next have arrived (only younger ones are left: loads arrive in the order in
  // which they were sent), and its reads are done; then the waves meet.  (A barrier alone does not wait for loads into LDS.)
  static __device__ __forceinline__ void meet() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kStages - 2) * (A::kLoads + B::kLoads)) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  }
  __device__ __forceinline__ void multiply(const u32x4 (&x)[TA], const u32x4 (&y)[TB]) {
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j) acc[i][j] = mma<T>(x[i], y[j], acc[i][j]);
  }
  static constexpr int kMine = A::Loads::kMine + B::Loads::kMine;
  __device__ __forceinline__ void start(char* into, int i) const {
    if (i < A::Loads::kMine) loads_a.start(sa, into, i);
    else if (i < kMine) loads_b.start(sb, into + A::kBytes, i - A::Loads::kMine);
  }
  // A step's products, x times y, and between them, one after each of the first products, the reads of the next step (kk of the
  // stage in `from`) and, with LOADS, the loads of the stage that comes: a wave has its SIMD to itself, so nothing is hidden but by
  // its own products, and the order is held as it stands here.
  template <bool PRODUCTS, bool LOADS>
  __device__ __forceinline__ void step(const u32x4 (&x)[TA], const u32x4 (&y)[TB], const char* from, int kk, u32x4 (&na)[TA], u32x4 (&nb)[TB],
                                       char* into) {
    constexpr int kMmas = TA * TB, kReads = TA + TB, kEarly = kMmas >= 2 ? kMmas / 2 : 1, kEach = (kReads + kEarly - 1) / kEarly;
    constexpr int kLoadEach = (kMine + kMmas - 1) / kMmas;
#pragma unroll
    for (int q = 0; q < kMmas; ++q) {
#pragma unroll
      for (int r = q * kEach; r < (q + 1) * kEach && r < kReads; ++r) {  // (the first of A, all of B, the others of A: as they are needed)
        if (r >= 1 && r <= TB) nb[r - 1] = B::fragment(from + A::kBytes, b0() + (r - 1) * 32, kk);
        else na[r == 0 ? 0 : r - TB] = A::fragment(from, a0() + (r == 0 ? 0 : r - TB) * 32, kk);
      }
      if constexpr (LOADS) {
#pragma unroll
        for (int i = q * kLoadEach; i < (q + 1) * kLoadEach && i < kMine; ++i) start(into, i);
      }
      if constexpr (PRODUCTS) {
        acc[q / TB][q % TB] = mma<T>(x[q / TB], y[q % TB], acc[q / TB][q % TB]);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  // Reads the stage in `from`, each step while the one before it is multiplied; `into`, which held the stage before, gets a new one.
  // (The two are never the same memory, and the compiler is told so: no read waits for the loads that are started here.)
  template <bool FIRST>
  __device__ __forceinline__ void stage(char* __restrict__ into, const char* __restrict__ from) {
    u32x4 na[TA], nb[TB];
    step<!FIRST, true>(fa, fb, from, 0, na, nb, into);
    next();
    step<true, false>(na, nb, from, 1, fa, fb, into);
#pragma unroll
    for (int kk = 2; kk < kSteps; kk += 2) {
      step<true, false>(fa, fb, from, kk, na, nb, into);
      step<true, false>(na, nb, from, kk + 1, fa, fb, into);
    }
  }

  // the first tile is at rows row_a, row_b; k from k0 to k1 (k1 > k0)
  __device__ __forceinline__ void begin(const Operand& op_a, const Operand& op_b, int64_t row_a, int64_t row_b, int64_t k0, int64_t k1, int step,
                                        char* lds_) {
    lds = lds_;
    step_rows = step;
    step_bytes = step * op_a.ld;
    left = stages = (int)((k1 - k0 + kK - 1) / kK);
    a = typename A::Place(op_a, row_a, k0);
    b = typename B::Place(op_b, row_b, k0);
    loads_a.begin(op_a, a);
    loads_b.begin(op_b, b);
    next_a = a;
    next_b = b;
    next_a.p += step_bytes;
    next_a.there -= step;
    if (step == 0) next_a.there = next_b.there = 0;  // (behind the only tile there is nothing to load)
    slot = kStages - 1;
    sa = loads_a.stage(a);
    sb = loads_b.stage(b);
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) {
#pragma unroll
      for (int i = 0; i < kMine; ++i) start(lds + s * kStage, i);
      next();
    }
  }
  // the next tile's product
  __device__ __forceinline__ void tile() {
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    int from = slot + 1 < kStages ? slot + 1 : 0;
    meet();
    stage<true>(lds + slot * kStage, lds + from * kStage);
    slot = from;
    for (int s = 1; s < stages; ++s) {
      from = slot + 1 < kStages ? slot + 1 : 0;
      meet();
      stage<false>(lds + slot * kStage, lds + from * kStage);
      slot = from;
    }
    multiply(fa, fb);
  }
  // LDS is free for other use: what is on its way has arrived, and all waves have read.  A block does not end without it.
  static __device__ __forceinline__ void end() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
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
  const int split = blockIdx.x % splits;
  const int64_t row0 = (int64_t)(blockIdx.x / splits) * P::kRowsB;
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

// a wave joins a row's splits
__global__ __launch_bounds__(kBlock) void k_xent_loss(const RowStat* __restrict__ part, int splits, int64_t n, int64_t vocab,
                                                      const int32_t* __restrict__ targets, int32_t ignore, float* __restrict__ loss,
                                                      float* __restrict__ lse, int32_t* __restrict__ bad) {
  const int64_t i = (int64_t)blockIdx.x * kWavesPerBlock + uniform_wave_in_block();
  if (i >= n) return;
  float m = kNoMax, sum = 0.f, target = 0.f;
  for (int s = lane_id(); s < splits; s += kWave) {
    const RowStat x = part[s * n + i];
    const float top = fmaxf(m, x.top);
    sum = sum * __builtin_amdgcn_exp2f(m - top) + x.sum * __builtin_amdgcn_exp2f(x.top - top);
    m = top;
    target += x.target;
  }
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1) {
    const float top = fmaxf(m, __shfl_xor(m, off, kWave)), mine = sum * __builtin_amdgcn_exp2f(m - top);
    sum = mine + __shfl_xor(mine, off, kWave);
    target += __shfl_xor(target, off, kWave);
    m = top;
  }
  if (lane_id() != 0) return;
  const int32_t t = targets[i];
  const bool ok = t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab;
  if (!ok && t != ignore) atomicOr(bad, 1);
  const float l = log2f(sum);
  lse[i] = (m + l) * kLn2;
  loss[i] = ok ? ((m - target) + l) * kLn2 : 0.f;
}

// ---- backward ------------------------------------------------------------------------------------------------------------
// What a row of G needs; target -1: the row has none, and G is zero there whatever its logits are.
struct RowTerm { float coef, lse2; int32_t target; int32_t pad; };

// In 16 bits G holds coef over the largest |coef| (and times 2^13 in fp16, whose exponents would otherwise not reach from 1 to a
// probability times dloss): where all rows count alike, as in a mean, the factor is 1 (a power of two), and so a target's p - 1 of a
// small p is not rounded away from -1 twice; with dloss itself in G, dH and dW of the mean were off by 3.0e-3 instead of 2.0e-3 (bf16).
template <bool LIFT>
__global__ __launch_bounds__(1024) void k_xent_terms(const int32_t* __restrict__ targets, int32_t ignore, const float* __restrict__ lse,
                                                     const float* __restrict__ dloss, float alpha, float most, int64_t n, int64_t rows, int64_t vocab,
                                                     RowTerm* __restrict__ term, float* __restrict__ unlift, int32_t* __restrict__ bad) {
  __shared__ float lds[16];
  float top = 0.f;
  if constexpr (LIFT) {  // (every block looks at all rows: no second launch, and n floats are little)
    for (int64_t i = threadIdx.x; i < n; i += 1024) {
      const int32_t t = targets[i];
      const float c = fabsf(alpha * dloss[i]);
      if (t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab && c < __builtin_inff()) top = fmaxf(top, c);
    }
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) top = fmaxf(top, __shfl_xor(top, off, kWave));
    if (lane_id() == 0) lds[wave_in_block()] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) top = fmaxf(top, lds[w]);
    if (top < 0x1p-100f) top = 0x1p-100f;
    if (top > 0x1p100f) top = 0x1p100f;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *unlift = LIFT ? top / most : 1.f;
  const int64_t i = (int64_t)blockIdx.x * 1024 + threadIdx.x;
  if (i >= rows) return;
  RowTerm r{0.f, 0.f, -1, 0};
  if (i < n) {
    const int32_t t = targets[i];
    const bool ok = t != ignore && (uint64_t)(int64_t)t < (uint64_t)vocab;
    if (ok) r = RowTerm{LIFT ? alpha * dloss[i] / top * most : alpha * dloss[i], lse[i] * kLog2e, t, 0};
    else if (t != ignore) atomicOr(bad, 1);
  }
  term[i] = r;
}

template <int T>
__device__ __forceinline__ void put4(char* p, const float (&f)[4]) {
  Pack<T, 4> x;
  x.set(f);
  x.store(p);
}

// G of the piece of the vocabulary that begins at v_first, [rows of H, ld bytes]; all of G's tiles are there, beyond the vocabulary's
// and the rows' end it is zero
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_g(Operand w, Operand h, int64_t vocab, int64_t k, float scale2, int64_t v_first,
                                                           uint32_t tiles_a, const RowTerm* __restrict__ term, char* __restrict__ g, int64_t ld) {
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> P;
  extern __shared__ char lds[];
  const int64_t piece0 = (int64_t)(blockIdx.x % tiles_a) * P::kRowsA, row0 = (int64_t)(blockIdx.x / tiles_a) * P::kRowsB;
  P p;
  p.begin(w, h, v_first + piece0, row0, 0, k, 0, lds);
  p.tile();
  P::end();
  const int first = (int)(v_first + piece0) + P::a0() + P::own_row(), left = (int)vocab - first;
  const bool ragged = v_first + piece0 + P::kRowsA > vocab;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t i = row0 + P::b0() + j * 32 + (lane_id() & 31);
    const RowTerm r = term[i];
    const int mine = r.target - first;
    const bool none = r.target < 0, hit = ballot64(!none && (uint32_t)mine < (uint32_t)(TA * 32)) != 0;
    char* to = g + i * ld + (piece0 + P::a0() + P::own_row()) * kElem<T>;
#pragma unroll
    for (int a = 0; a < TA; ++a) {
      f32x16 x = p.acc[a][j];
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[e], scale2, -r.lse2));
      if (hit) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (!none && mine == a * 32 + P::row_of(e)) x[e] -= 1.f;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) x[e] = none ? 0.f : x[e] * r.coef;
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

// dH: sums[split][row][dim] (+)= the split's part of G W over the piece
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_dh(Operand wt, Operand g, int64_t k, int splits, uint32_t tiles_a, uint32_t tiles_b,
                                                            bool add, float* __restrict__ sums, int64_t width) {
  typedef Product<T, WA, WB, TA, TB, true, false, kWide> P;
  extern __shared__ char lds[];
  const uint32_t tile = blockIdx.x / splits, split = blockIdx.x % splits;
  const int64_t col0 = (int64_t)(tile % tiles_a) * P::kRowsA, row0 = (int64_t)(tile / tiles_a) * P::kRowsB;
  const int64_t stages = (k + P::kK - 1) / P::kK;
  const int64_t k0 = stages * split / splits * P::kK, k1 = stages * (split + 1) / splits * P::kK;
  P p;
  p.begin(wt, g, col0, row0, k0, k1, 0, lds);
  p.tile();
  P::end();
  float* to = sums + (int64_t)split * tiles_b * P::kRowsB * width;
#pragma unroll
  for (int j = 0; j < TB; ++j)
#pragma unroll
    for (int a = 0; a < TA; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t c = col0 + P::a0() + P::own_row() + a * 32 + P::row_of(4 * q);
        if (c >= width) continue;
        float* at = to + (row0 + P::b0() + j * 32 + (lane_id() & 31)) * width + c;
        f32x16& x = p.acc[a][j];
        u32x4 old = add ? *reinterpret_cast<const u32x4*>(at) : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) old[e] = __float_as_uint(__uint_as_float(old[e]) + x[4 * q + e]);
        *reinterpret_cast<u32x4*>(at) = old;
      }
}

template <int T>
__global__ __launch_bounds__(kBlock) void k_xent_dh_out(const float* __restrict__ sums, int splits, int64_t rows, int64_t width, int64_t n,
                                                        int32_t dim, const float* __restrict__ unlift, char* __restrict__ out) {
  const int64_t step = (int64_t)gridDim.x * kBlock;
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < n * dim; i += step) {
    const int64_t row = i / dim;
    const int32_t c = (int32_t)(i - row * dim);
    float s = 0.f;
    for (int q = 0; q < splits; ++q) s += sums[((int64_t)q * rows + row) * width + c];
    ((typename Element<T>::M*)out)[i] = (typename Element<T>::M)(s * *unlift);
  }
}

// dW of the piece: rows v_first .. of the weight's gradient
template <int T, int WA, int WB, int TA, int TB>
__global__ __launch_bounds__(WA* WB* kWave) __attribute__((amdgpu_waves_per_eu(1))) void k_xent_dw(Operand ht, Operand gt, int64_t k, int64_t vocab, int64_t v_first, int32_t dim,
                                                            uint32_t tiles_a, const float* __restrict__ unlift, char* __restrict__ out) {
  typedef Product<T, WA, WB, TA, TB, true, true, kNarrow> P;
  extern __shared__ char lds[];
  const int64_t col0 = (int64_t)(blockIdx.x % tiles_a) * P::kRowsA, piece0 = (int64_t)(blockIdx.x / tiles_a) * P::kRowsB;
  P p;
  p.begin(ht, gt, col0, piece0, 0, k, 0, lds);
  p.tile();
  P::end();
  const float u = *unlift;
#pragma unroll
  for (int j = 0; j < TB; ++j) {
    const int64_t v = v_first + piece0 + P::b0() + j * 32 + (lane_id() & 31);
    if (v >= vocab) continue;
#pragma unroll
    for (int a = 0; a < TA; ++a)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t c = col0 + P::a0() + P::own_row() + a * 32 + P::row_of(4 * q);
        float f[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = p.acc[a][j][4 * q + e] * u;
        if (c + 4 <= dim) {
          put4<T>(out + (v * dim + c) * kElem<T>, f);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (c + e < dim) ((typename Element<T>::M*)out)[v * dim + c + e] = (typename Element<T>::M)f[e];
        }
      }
  }
}

// rows of `dim` elements into rows of `ld` bytes, what is behind a row's end zero
template <int T>
__global__ __launch_bounds__(kBlock) void k_xent_pad(const char* __restrict__ in, int64_t rows, int32_t dim, char* __restrict__ out, int32_t width) {
  const int64_t step = (int64_t)gridDim.x * kBlock;
  for (int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x; i < rows * width; i += step) {
    const int64_t row = i / width;
    const int32_t c = (int32_t)(i - row * width);
    typedef typename Element<T>::M M;
    ((M*)out)[i] = c < dim ? ((const M*)in)[row * dim + c] : (M)0.f;
  }
}

// ---- the workspace ---------------------------------------------------------------------------------------------------------
constexpr int64_t kPieceBytes = (int64_t)256 << 20;  // of G
constexpr int64_t kMaxVocab = 0x7FFFF000;            // (a tile's row numbers stay below 2^31)
constexpr int kTile = 256;                            // rows of a block's tile, either way

int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

struct XentPlan {
  int64_t n, vocab, width, ld;  // width: elements of a padded row
  int64_t rows, piece, pieces;
  int64_t g_ld;  // bytes from row to row of G: not a power of two, or a tile's rows would all lie in the same few channels of memory
  int splits, dh_splits;
  bool few, pad;
  size_t h, w, part, term, unlift, g, sums, bytes;
  XentPlan(int64_t n_, int64_t vocab_, int32_t dim, int dtype, bool aligned, bool grad) : n(n_), vocab(vocab_) {
    const int es = element_bytes(dtype);
    width = round_up(dim, 16 / es);
    ld = width * es;
    pad = !aligned || width != dim;
    few = n <= 32;
    rows = round_up(n, kTile);
    const int64_t row_tiles = few ? 1 : rows / kTile, vocab_tiles = (vocab + kTile - 1) / kTile;
    int64_t s = (few ? 1024 : 256) / row_tiles;
    s = s < 1 ? 1 : s;
    splits = (int)(s < vocab_tiles ? s : vocab_tiles);
    piece = kPieceBytes / (rows * es) / kTile * kTile;
    if (piece < kTile) piece = kTile;
    if (piece > vocab_tiles * kTile) piece = vocab_tiles * kTile;
    pieces = (vocab + piece - 1) / piece;
    const int64_t dh_tiles = rows / kTile * ((width + kTile - 1) / kTile);
    int64_t ds = 256 / dh_tiles;
    const int64_t first = piece < vocab ? piece : vocab, stages = (first * es + kWide - 1) / kWide;
    ds = ds < 1 ? 1 : ds > 16 ? 16 : ds;
    dh_splits = (int)(ds < stages ? ds : stages);
    size_t at = 0;
    auto take = [&](size_t b) { const size_t o = at; at += (b + 255) & ~(size_t)255; return o; };
    h = take(pad ? (size_t)n * ld : 0);
    w = take(pad ? (size_t)vocab * ld : 0);
    part = take(grad ? 0 : (size_t)splits * n * sizeof(RowStat));
    term = take(grad ? (size_t)rows * sizeof(RowTerm) : 0);
    unlift = take(grad ? sizeof(float) : 0);
    g_ld = piece * es + 256;
    g = take(grad ? (size_t)rows * g_ld : 0);
    sums = take(grad ? (size_t)dh_splits * rows * width * sizeof(float) : 0);
    bytes = at + 256;
  }
};

template <int T>
void pad_rows(const void* in, int64_t rows, int32_t dim, const XentPlan& p, void* out, hipStream_t s) {
  const int64_t blocks = (rows * p.width + kBlock - 1) / kBlock;
  COOP_LAUNCH(K_XENT_PAD, k_xent_pad<T>, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(kBlock), 0, s, (const char*)in, rows, dim, (char*)out,
              (int32_t)p.width);
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

template <int T, int WA, int WB, int TA, int TB>
bool launch_stats(const XentPlan& p, Operand w, Operand h, float alpha, const int32_t* targets, RowStat* part, hipStream_t s) {
  typedef Product<T, WA, WB, TA, TB, false, false, kWide> P;
  constexpr int lds = P::kLds > WA * P::kRowsB * (int)sizeof(RowStat) ? P::kLds : WA * P::kRowsB * (int)sizeof(RowStat);
  const auto kernel = k_xent_stats<T, WA, WB, TA, TB>;
  if (!allow_lds(kernel, lds)) return false;
  const int64_t row_tiles = (p.n + P::kRowsB - 1) / P::kRowsB;
  COOP_LAUNCH(K_XENT_STATS, kernel, dim3((unsigned)(row_tiles * p.splits)), dim3(P::kThreads), lds, s, w, h, p.n, p.vocab, p.width, alpha * kLog2e,
              targets, p.splits, part);
  return true;
}

template <int T>
int forward(const XentPlan& p, const void* hidden, const void* weight, int32_t dim, const int32_t* targets, float alpha, int32_t ignore,
            float* loss, float* lse, char* ws, int32_t* bad, hipStream_t s) {
  if (p.pad) {
    pad_rows<T>(hidden, p.n, dim, p, ws + p.h, s);
    pad_rows<T>(weight, p.vocab, dim, p, ws + p.w, s);
    hidden = ws + p.h;
    weight = ws + p.w;
  }
  const Operand w{(const char*)weight, p.ld, p.vocab, p.ld}, h{(const char*)hidden, p.ld, p.n, p.ld};
  RowStat* part = (RowStat*)(ws + p.part);
  const bool ok = p.few ? launch_stats<T, 4, 1, 2, 1>(p, w, h, alpha, targets, part, s) : launch_stats<T, 2, 2, 4, 4>(p, w, h, alpha, targets, part, s);
  if (!ok) return COOP_E_HIP;
  COOP_LAUNCH(K_XENT_LOSS, k_xent_loss, dim3((unsigned)((p.n + kWavesPerBlock - 1) / kWavesPerBlock)), dim3(kBlock), 0, s, (const RowStat*)part, p.splits, p.n,
              p.vocab, targets, ignore, loss, lse, bad);
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

template <int T>
int backward(const XentPlan& p, const void* hidden, const void* weight, int32_t dim, const int32_t* targets, float alpha, int32_t ignore,
             const float* lse, const float* dloss, void* dhidden, void* dweight, char* ws, int32_t* bad, hipStream_t s) {
  if (p.pad) {
    pad_rows<T>(hidden, p.n, dim, p, ws + p.h, s);
    pad_rows<T>(weight, p.vocab, dim, p, ws + p.w, s);
    hidden = ws + p.h;
    weight = ws + p.w;
  }
  RowTerm* term = (RowTerm*)(ws + p.term);
  float* unlift = (float*)(ws + p.unlift);
  char* g = ws + p.g;
  float* sums = (float*)(ws + p.sums);
  COOP_LAUNCH(K_XENT_TERMS, (k_xent_terms<T != COOP_F32>), dim3((unsigned)((p.rows + 1023) / 1024)), dim3(1024), 0, s, targets, ignore, lse, dloss,
              alpha, T == COOP_F16 ? 8192.f : 1.f, p.n, p.rows, p.vocab, term, unlift, bad);
  const int64_t g_ld = p.g_ld;
  const Operand w{(const char*)weight, p.ld, p.vocab, p.ld}, h{(const char*)hidden, p.ld, p.n, p.ld};
  typedef Product<T, 2, 2, 4, 4, false, false, kWide> P;
  const auto kg = k_xent_g<T, 2, 2, 4, 4>;
  const auto kh = k_xent_dh<T, 2, 2, 4, 4>;
  const auto kw = k_xent_dw<T, 2, 2, 4, 4>;
  if (!allow_lds(kg, P::kLds) || !allow_lds(kh, P::kLds) || !allow_lds(kw, P::kLds)) return COOP_E_HIP;
  const uint32_t row_tiles = (uint32_t)(p.rows / kTile), col_tiles = (uint32_t)((p.width + kTile - 1) / kTile);
  for (int64_t v = 0; v < p.vocab; v += p.piece) {
    const int64_t len = p.vocab - v < p.piece ? p.vocab - v : p.piece;
    const uint32_t tiles = (uint32_t)((len + kTile - 1) / kTile);
    COOP_LAUNCH(K_XENT_G, kg, dim3(tiles * row_tiles), dim3(P::kThreads), P::kLds, s, w, h, p.vocab, p.width, alpha * kLog2e, v, tiles,
                (const RowTerm*)term, g, g_ld);
    if (dhidden != nullptr) {
      const Operand wt{(const char*)weight + v * p.ld, p.ld, p.ld, len}, gi{g, g_ld, p.rows, (int64_t)tiles * kTile * kElem<T>};
      // (every split has something to do: the last piece may be too short for all of them, and then adds nothing to the others' sums)
      const int64_t stages = (len + P::kK - 1) / P::kK;
      const int splits = (int)(p.dh_splits < stages ? p.dh_splits : stages);
      COOP_LAUNCH(K_XENT_DH, kh, dim3(row_tiles * col_tiles * splits), dim3(P::kThreads), P::kLds, s, wt, gi, len, splits, col_tiles, row_tiles,
                  v != 0, sums, p.width);
    }
    if (dweight != nullptr) {
      const Operand ht{(const char*)hidden, p.ld, p.ld, p.n}, gt{g, g_ld, (int64_t)tiles * kTile * kElem<T>, p.rows};
      COOP_LAUNCH(K_XENT_DW, kw, dim3(tiles * col_tiles), dim3(P::kThreads), P::kLds, s, ht, gt, p.n, p.vocab, v, dim, col_tiles,
                  (const float*)unlift, (char*)dweight);
    }
  }
  const int64_t out_blocks = (p.n * dim + kBlock - 1) / kBlock;
  if (dhidden != nullptr)
    COOP_LAUNCH(K_XENT_DH_OUT, k_xent_dh_out<T>, dim3((unsigned)(out_blocks < 16384 ? out_blocks : 16384)), dim3(kBlock), 0, s, (const float*)sums,
                p.dh_splits, p.rows, p.width, p.n, dim, (const float*)unlift, (char*)dhidden);
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
