// Products on the matrix units: C = A B^T over a common dimension k, from tiles of both operands in LDS.
//
// An operand either has k as its contiguous dimension (rows of 64 or 128 bytes of k per stage) or as its row number (then its fragments
// are transposed on the way from LDS to the registers).  The columns of C, rows of B, lie on the lanes; its rows, rows of A, in a lane's
// registers.
#pragma once
#include "elements.h"

namespace coop {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char LdsByte;

// Bytes of k per row and stage: 64 (32 elements of 16 bits, 16 of 32), four stages in LDS, or 128, two of them.  One is read, the others
// are on their way.  Rows of 64 bytes are half a cache line, so operands with k contiguous take 128.
constexpr int kWide = 128, kNarrow = 64;
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
  int64_t other = 0;  // of a pair, or of two parts that are added up: bytes from this one to the other
};

// How a stage of R rows of an operand lies in LDS, in 16-byte slots filled in order by the loads, 64 to a wave's load.
//   k contiguous: a row's 4 or 8 chunks, exchanged by the row's number so that what 8 or 16 lanes read together lies in different banks;
//   k strided: a row of k holds R elements; its chunks are exchanged by k so that what one fragment reads lies in different banks.
// Both exchanges are an exclusive or with bits that neither the next tile of 32 rows nor the next step of k changes.
// PAIR: the rows are those of two operands of one shape, 32 of the one and the same 32 of the other in turn; rows are counted in either.
template <int T, int R, bool STRIDED, int SIZE, int WAVES, bool PAIR = false>
struct Staged {
  static_assert(!PAIR || (!STRIDED && R % 64 == 0 && 64 * 16 * WAVES == 32 * SIZE), "a load of all waves has 32 rows of one of the two");
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
    int64_t other;  // PAIR: from one operand to the other
    int there, in_row;
    __device__ __forceinline__ Place() {}
    __device__ __forceinline__ Place(const Operand& op, int64_t row0, int64_t k0) {
      const int64_t most = 0x7FFFFFFF, rows = STRIDED ? op.k - k0 : op.rows - row0, bytes = STRIDED ? op.rows - row0 * kElem<T> : op.k - k0 * kElem<T>;
      p = op.base + (STRIDED ? k0 * op.ld + row0 * kElem<T> : row0 * op.ld + k0 * kElem<T>);
      other = PAIR ? op.other : 0;
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
        at[i] = (PAIR ? (row >> 6) * 32 + (row & 31) : row) * ld + chunk;
        if (STRIDED && chunk >= first.in_row) at[i] = kNowhere;
      }
    }
    // what the loads of a stage have in common
    struct Stage {
      __amdgpu_buffer_rsrc_t rsrc, rsrc2;
      int off;
    };
    __device__ __forceinline__ Stage stage(const Place& s) const {
      constexpr int kRows = STRIDED ? kK : PAIR ? R / 2 : R;
      const int rows = s.there < kRows ? s.there : kRows, in_row = s.in_row < ld ? s.in_row : ld, last = (rows - 1) * ld + in_row;
      const int records = (rows < in_row ? rows : in_row) > 0 ? last : 0;
      return Stage{__builtin_amdgcn_make_buffer_rsrc((void*)s.p, 0, records, 0x00020000),
                   __builtin_amdgcn_make_buffer_rsrc((void*)(s.p + (PAIR ? s.other : 0)), 0, records, 0x00020000), !STRIDED && chunk >= s.in_row ? kNowhere : 0};
    }
    __device__ __forceinline__ void start(const Stage& s, char* lds, int i) const {
      const int l = i * WAVES + uniform_wave_in_block();
      if (kAll < WAVES && l >= kAll) return;
      const int at_lds = l * 1024, from = STRIDED ? at[i] : at[i] + s.off;
      if (PAIR && (i & 1) != 0) {  // (a load has rows of one of the two, and all waves of the same)
        __builtin_amdgcn_raw_ptr_buffer_load_lds(s.rsrc2, (__attribute__((address_space(3))) void*)(LdsByte*)(lds + at_lds), 16, from, 0, 0, 0);
        return;
      }
      __builtin_amdgcn_raw_ptr_buffer_load_lds(s.rsrc, (__attribute__((address_space(3))) void*)(LdsByte*)(lds + at_lds), 16, from, 0, 0, 0);
    }
  };
  // the fragment of rows row .. row + 31 at step kk of the stage
  static __device__ __forceinline__ u32x4 fragment(const char* lds, int row, int kk, int lane = lane_id()) {
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
// TWICE: B is the sum of two operands of one layout, and every stage of A is multiplied by both of its stages of B, one after the other (A's comes from L2
// the second time).
template <int T, int WA, int WB, int TA, int TB, bool SA, bool SB, int SIZE, bool PAIR = false, bool TWICE = false>
struct Product {
  static constexpr int kWaves = WA * WB, kThreads = kWaves * kWave;
  static constexpr int kRowsA = WA * TA * 32, kRowsB = WB * TB * 32;
  static constexpr int kK = SIZE / kElem<T>, kSteps = SIZE / 32, kStages = 256 / SIZE, kTimes = TWICE ? 2 : 1;
  typedef Staged<T, kRowsA, SA, SIZE, kWaves, PAIR> A;
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
  int64_t to_rest;              // TWICE: bytes from B to what is added to it
  char* lds;

  __device__ __forceinline__ static int a0() { return uniform_wave_in_block() / WB * (TA * 32); }
  __device__ __forceinline__ static int b0() { return uniform_wave_in_block() % WB * (TB * 32); }
  // C's element j of a 32 x 32 tile: its row is the lane's own plus one that all lanes have; its column is lane & 31
  __device__ __forceinline__ static int own_row() { return (lane_id() >> 5) * 4; }
  __device__ __forceinline__ static constexpr int row_of(int j) { return (j >> 2) * 8 + (j & 3); }

  // to the next stage of the stream
  __device__ __forceinline__ void next() {
    if constexpr (TWICE) {
      if ((left-- & 1) == 0) {  // (an even number are left ahead of a stage's first time)
        b.p += to_rest;
        sb = loads_b.stage(b);
        return;
      }
      b.p -= to_rest;
      ++left;
    }
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
    to_rest = op_b.other;
    left = stages = (int)((k1 - k0 + kK - 1) / kK) * kTimes;
    a = typename A::Place(op_a, row_a, k0);
    b = typename B::Place(op_b, row_b, k0);
    loads_a.begin(op_a, a);
    loads_b.begin(op_b, b);
    next_a = a;
    next_b = b;
    next_a.p += step_bytes;
    next_a.there -= step;
    if (step == 0) next_a.there = next_b.there = 0;  // (behind the only tile there is nothing to load)
    start_stream();
  }
  // The same for one tile whose k has two parts, of operands of their own and as long as each other: tile(), last(), tile().
  __device__ __forceinline__ void begin_two(const Operand& op_a, const Operand& op_b, const Operand& then_a, const Operand& then_b, int64_t row_a,
                                            int64_t row_b, int64_t k0, int64_t k1, char* lds_) {
    lds = lds_;
    step_rows = 0;
    step_bytes = 0;
    to_rest = op_b.other;
    left = stages = (int)((k1 - k0 + kK - 1) / kK) * kTimes;
    a = typename A::Place(op_a, row_a, k0);
    b = typename B::Place(op_b, row_b, k0);
    loads_a.begin(op_a, a);
    loads_b.begin(op_b, b);
    next_a = typename A::Place(then_a, row_a, k0);
    next_b = typename B::Place(then_b, row_b, k0);
    start_stream();
  }
  // What is loaded next is the second part's, from its second stage on: behind it there is nothing to load.
  __device__ __forceinline__ void last() {
    next_a.there = next_b.there = 0;
    if (left == stages) {  // (it has one stage)
      a.there = b.there = 0;
      sa = loads_a.stage(a);
      sb = loads_b.stage(b);
    }
  }
  __device__ __forceinline__ void start_stream() {
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
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < TA; ++i)
#pragma unroll
      for (int j = 0; j < TB; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  }
  // the next tile's product, added to acc
  __device__ __forceinline__ void tile() {
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

}  // namespace coop
