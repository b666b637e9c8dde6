// Learned rows: out[i, :] = s_i E[ids[i], :] with s_i = alpha scale[i], and the way back,
// dE[v, :] = sum over the tokens i with ids[i] = v of s_i dout[i, :].
//
// Both are bound by HBM: every row is read once and every output row written once.
#include <type_traits>

#include "coop_internal.h"
#include "elements.h"

namespace coop {
namespace {

// ---- lookup ------------------------------------------------------------------------------------------------------------
// The rows' items (E elements each, the last one anchored at the row's end) are dealt to the threads in order, four in flight each.
// 2,592,327 rows of 128 elements of fp16 out of 7.1 GB: 236 us, 1.35 GB at 5.7 TB/s; 24 rows of 100: 2.5 us, a wait for memory or two.
constexpr int kUnroll = 4;

// An id that has no row is reported unless it is the one that says so; COOP_NO_PAD says that there is none, and is no id itself.
__device__ __forceinline__ bool wrong_id(int32_t id, int32_t pad) { return id != pad || pad == COOP_NO_PAD; }

struct EmbedShape {
  int64_t n_rows, n_ids;
  int32_t dim, pad;
  uint32_t vecs, magic;  // items per row, ceil(2^32 / vecs)
};

template <int TI, int TO, int E>
__global__ __launch_bounds__(kBlock) void k_embed(const char* __restrict__ table, EmbedShape sh, const int32_t* __restrict__ ids,
                                                  const float* __restrict__ scale, float alpha, char* __restrict__ out,
                                                  int32_t* __restrict__ bad) {
  typedef Pack<TI, E> In;
  typedef Pack<TO, E> Out;
  const RowShape rs{0, sh.vecs, sh.magic, 0};
  const BlockItems items((int64_t)blockIdx.x * (kBlock * kUnroll), sh.vecs);
  int64_t row[kUnroll];
  int32_t id[kUnroll];
  float s[kUnroll];
  int32_t col[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    uint32_t item;
    row[u] = items.row_of((uint32_t)(u * kBlock) + threadIdx.x, rs, &item);
    const int64_t r = row[u] < sh.n_ids ? row[u] : sh.n_ids - 1;
    id[u] = ids[r];
    s[u] = scale != nullptr ? scale[r] * alpha : alpha;
    const int64_t c = (int64_t)item * E, last = sh.dim - E;
    col[u] = (int32_t)(c < last ? c : last);
  }
  In x[kUnroll];
  bool ok[kUnroll];
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    ok[u] = id[u] != sh.pad && (uint64_t)(int64_t)id[u] < (uint64_t)sh.n_rows;
    // (every load is issued, without a branch: that of a place without a row reads row 0)
    x[u] = In::load(table + ((ok[u] ? (int64_t)id[u] : 0) * sh.dim + col[u]) * (int64_t)sizeof(typename In::M));
  }
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    if (row[u] >= sh.n_ids) continue;
    float f[E];
    x[u].get(f);
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = ok[u] ? f[e] * s[u] : 0.f;
    Out y;
    y.set(f);
    y.store_nt(out + (row[u] * sh.dim + col[u]) * (int64_t)sizeof(typename Out::M));
    if (!ok[u] && wrong_id(id[u], sh.pad) && col[u] == 0) atomicOr(bad, 1);
  }
}

// ---- the tokens in the order of their ids ------------------------------------------------------------------------------
// A stable radix sort of (id, place), 8 bits at a time, least significant first.  Per pass the digits of every tile are counted, and then
// every tile goes to its places: tokens of the digits in front, and of the same digit in the tiles in front.  A block of the second kernel
// adds these up from the counts itself (up to kOwnTiles of them; above that a scan does).  Inside a tile a wave ranks its tokens 64 at a
// time: the lanes with the same digit are found by a ballot per bit, and a counter per wave and digit holds how many came before; the
// tile is brought into its order in LDS, so that tokens of a digit, some 32 of them, leave side by side.  A place without a row has the
// key n_rows and comes last.  Up to 8,192 tokens one block does all passes, the tokens in its LDS between them.
//
// A million ids of 22 bits: 72 us, three passes of 9 and 15; 138 us in three of count, scan and unordered stores, 125 us in two of 11 bits
// (the runs of a digit are then 4 tokens, and single stores to memory go at 80 a nanosecond at best).  Bound by the 125 blocks' own chain of
// reads, ballots and barriers: the bytes, 16 a token and pass, would take 7 us.
constexpr int kKeysPerThread = 8;
constexpr int kSortBlock = 1024;
constexpr int kSortWaves = kSortBlock / kWave;
constexpr int kSortTile = kSortBlock * kKeysPerThread;
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;
constexpr int64_t kOwnTiles = 512;

// The zeros of a dense gradient, written by blocks of the sort's launches behind those that sort: a launch less where there are few (76 -> 71
// us for 50,021 rows of 75), and where there are many the sort goes on beside them (944 MB and 3,853 tokens: 230 -> 199 us, sums and all).  In pieces of
// 16 bytes; `head` bytes in front of the first and `tail` behind the last, 2 a thread.
struct Zeros {
  char* p;
  int64_t head, pieces, tail;
  __device__ __forceinline__ void write(uint32_t block, uint32_t blocks) const {
    const int64_t stride = (int64_t)blocks * blockDim.x;
    const u32x4 zero = {0, 0, 0, 0};
#pragma unroll 4
    for (int64_t i = (int64_t)block * blockDim.x + threadIdx.x; i < pieces; i += stride) reinterpret_cast<u32x4*>(p + head)[i] = zero;
    if (block != 0 || threadIdx.x >= 8) return;
    if (2 * (int64_t)threadIdx.x < head) reinterpret_cast<uint16_t*>(p)[threadIdx.x] = 0;
    if (2 * (int64_t)threadIdx.x < tail) reinterpret_cast<uint16_t*>(p + head + 16 * pieces)[threadIdx.x] = 0;
  }
  // part i of `of`
  Zeros part(int i, int of) const {
    const int64_t from = pieces * i / of, to = pieces * (i + 1) / of;
    return Zeros{i == 0 ? p : p + head + 16 * from, i == 0 ? head : 0, to - from, i + 1 == of ? tail : 0};
  }
  uint32_t blocks(int threads) const {  // some four pieces a thread
    const int64_t b = (pieces + 4 * threads - 1) / (4 * threads);
    return (uint32_t)(b > 16384 ? 16384 : b < 1 && head + tail > 0 ? 1 : b);
  }
};
Zeros zeros_of(void* p, int64_t bytes) {
  int64_t head = (int64_t)((16 - ((uintptr_t)p & 15)) & 15);
  if (head > bytes) head = bytes;
  const int64_t pieces = (bytes - head) / 16;
  return Zeros{(char*)p, head, pieces, bytes - head - 16 * pieces};
}

struct SortInput {  // the first pass reads the ids, the others the (key, place) pairs that the pass before has left
  const int32_t* ids;
  const u32x2* pairs;
  int64_t n_rows;
  int32_t pad;
  __device__ __forceinline__ u32x2 at(int64_t i, bool* wrong) const {
    if (ids == nullptr) return pairs[i];
    const int32_t id = ids[i];
    const bool row = id != pad && (uint64_t)(int64_t)id < (uint64_t)n_rows;
    *wrong |= !row && wrong_id(id, pad);
    return u32x2{row ? (uint32_t)id : (uint32_t)n_rows, (uint32_t)i};
  }
};

// matrix: [tile][digit], or [digit][tile] for a scan
template <bool OWN>
__global__ __launch_bounds__(kSortBlock) void k_sort_count(SortInput in, int64_t n, int shift, uint32_t* __restrict__ matrix, uint32_t tiles,
                                                           int32_t* __restrict__ bad, Zeros zeros) {
  if (blockIdx.x >= tiles) return zeros.write(blockIdx.x - tiles, gridDim.x - tiles);
  __shared__ uint32_t cnt[kDigits];
  if (threadIdx.x < kDigits) cnt[threadIdx.x] = 0;
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  bool wrong = false;
  uint32_t key[kKeysPerThread];
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const int64_t i = base + u * kSortBlock + threadIdx.x;
    key[u] = i < n ? in.at(i, &wrong)[0] : 0u;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u)
    if (base + u * kSortBlock + threadIdx.x < n) atomicAdd(&cnt[key[u] >> shift & (kDigits - 1)], 1u);
  if (wrong) atomicOr(bad, 1);
  __syncthreads();
  if (threadIdx.x < kDigits) matrix[OWN ? (size_t)blockIdx.x * kDigits + threadIdx.x : (size_t)threadIdx.x * tiles + blockIdx.x] = cnt[threadIdx.x];
}

// LDS of a block that brings its tokens into order
struct SortLds {
  u32x2 pair[kSortTile];
  uint16_t cnt[kSortWaves][kDigits];
  uint32_t local[kDigits];  // the block's tokens of the digits in front
  uint32_t sums[kSortWaves];
  uint32_t parts[2][kSortBlock];
};

// exclusive sums over the digits, a thread of the first kDigits for each
__device__ __forceinline__ uint32_t digit_offset(uint32_t mine, SortLds* lds) {
  uint32_t upto = 0;
  __syncthreads();
  if (threadIdx.x < kDigits) {
    upto = wave_incl_scan(mine);
    if (lane_id() == kWave - 1) lds->sums[wave_in_block()] = upto;
  }
  __syncthreads();
  uint32_t at = upto - mine;
  if (threadIdx.x < kDigits)
    for (int w = 0; w < wave_in_block(); ++w) at += lds->sums[w];
  return at;
}

// A thread's tokens into the block's LDS in the order of the digit
__device__ __forceinline__ void order_block(const u32x2 (&x)[kKeysPerThread], const bool (&live)[kKeysPerThread], int shift, SortLds* lds) {
  for (int d = threadIdx.x; d < kDigits * kSortWaves / 2; d += kSortBlock) reinterpret_cast<uint32_t*>(lds->cnt)[d] = 0;
  __syncthreads();
  uint16_t* cnt = lds->cnt[uniform_wave_in_block()];
  uint32_t rank[kKeysPerThread];
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const uint32_t d = x[u][0] >> shift & (kDigits - 1);
    uint64_t same = ballot64(live[u]);
#pragma unroll
    for (int b = 0; b < kDigitBits; ++b) {
      const uint64_t set = ballot64(d >> b & 1);
      same &= d >> b & 1 ? set : ~set;
    }
    const uint32_t before = lanes_below(same), ran = cnt[d];
    rank[u] = ran + before;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (live[u] && before == 0) cnt[d] = (uint16_t)(ran + (uint32_t)__popcll(same));
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t all = 0;
  if (threadIdx.x < kDigits) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) all += lds->cnt[w][threadIdx.x];
  }
  uint32_t at = digit_offset(all, lds);
  if (threadIdx.x < kDigits) {
    lds->local[threadIdx.x] = at;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = lds->cnt[w][threadIdx.x];
      lds->cnt[w][threadIdx.x] = (uint16_t)at;  // (below the tile's 8,192 tokens)
      at += c;
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u)
    if (live[u]) lds->pair[cnt[x[u][0] >> shift & (kDigits - 1)] + rank[u]] = x[u];
  __syncthreads();
}

// counts: OWN, the matrix [tile][digit]; else its scan [digit][tile].  The last pass leaves keys and places apart.
template <bool OWN>
__global__ __launch_bounds__(kSortBlock) void k_sort_place(SortInput in, int64_t n, int shift, const uint32_t* __restrict__ counts, uint32_t tiles,
                                                           u32x2* __restrict__ pairs_out, uint32_t* __restrict__ keys_out,
                                                           uint32_t* __restrict__ places_out, Zeros zeros) {
  if (blockIdx.x >= tiles) return zeros.write(blockIdx.x - tiles, gridDim.x - tiles);
  extern __shared__ char sort_lds[];
  SortLds* lds = reinterpret_cast<SortLds*>(sort_lds);
  const int64_t first = (int64_t)blockIdx.x * kSortTile, base = first + uniform_wave_in_block() * (kKeysPerThread * kWave) + lane_id();
  u32x2 x[kKeysPerThread];
  bool live[kKeysPerThread], unused = false;
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    live[u] = base + u * kWave < n;
    x[u] = live[u] ? in.at(base + u * kWave, &unused) : u32x2{0, 0};
  }
  uint32_t from = 0;  // of digit threadIdx.x: where its tokens of this tile begin
  if constexpr (OWN) {
    constexpr int kParts = kSortBlock / kDigits;
    const uint32_t d = threadIdx.x & (kDigits - 1), part = threadIdx.x / kDigits;
    uint32_t in_front = 0, all = 0;
#pragma unroll 8
    for (uint32_t t = part; t < tiles; t += kParts) {
      const uint32_t c = counts[(size_t)t * kDigits + d];
      all += c;
      in_front += t < blockIdx.x ? c : 0;
    }
    lds->parts[0][threadIdx.x] = in_front;
    lds->parts[1][threadIdx.x] = all;
    __syncthreads();
    in_front = all = 0;
#pragma unroll
    for (int p = 0; p < kParts; ++p) {
      in_front += lds->parts[0][p * kDigits + d];
      all += lds->parts[1][p * kDigits + d];
    }
    from = in_front + digit_offset(all, lds);
  } else if (threadIdx.x < kDigits) {
    from = counts[(size_t)threadIdx.x * tiles + blockIdx.x];
  }
  order_block(x, live, shift, lds);
  if (threadIdx.x < kDigits) lds->parts[0][threadIdx.x] = from - lds->local[threadIdx.x];
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const int at = u * kSortBlock + threadIdx.x;
    if (first + at >= n) break;
    const u32x2 p = lds->pair[at];
    const uint32_t to = lds->parts[0][p[0] >> shift & (kDigits - 1)] + at;
    if (keys_out == nullptr) {
      pairs_out[to] = p;
    } else {
      keys_out[to] = p[0];
      places_out[to] = p[1];
    }
  }
}

// n <= kSortTile: all passes, and where the rows form's rows go (RowPlaces: of one tile of chunks)
__global__ __launch_bounds__(kSortBlock) void k_sort_small(SortInput in, int n, int bits, uint32_t* __restrict__ keys_out,
                                                           uint32_t* __restrict__ places_out, uint32_t* __restrict__ in_tile,
                                                           uint32_t* __restrict__ total, int32_t* __restrict__ bad, Zeros zeros) {
  if (blockIdx.x != 0) return zeros.write(blockIdx.x - 1, gridDim.x - 1);
  extern __shared__ char sort_lds[];
  SortLds* lds = reinterpret_cast<SortLds*>(sort_lds);
  const int base = uniform_wave_in_block() * (kKeysPerThread * kWave) + lane_id();
  u32x2 x[kKeysPerThread];
  bool live[kKeysPerThread], wrong = false;
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    live[u] = base + u * kWave < n;
    x[u] = live[u] ? in.at(base + u * kWave, &wrong) : u32x2{0, 0};
  }
  if (wrong) atomicOr(bad, 1);
  for (int shift = 0; shift < bits; shift += kDigitBits) {
    order_block(x, live, shift, lds);
#pragma unroll
    for (int u = 0; u < kKeysPerThread; ++u)
      if (live[u]) x[u] = lds->pair[base + u * kWave];
  }
  // a wave's 512 tokens are 16 chunks: the rows that begin in each, and in front of it
  uint32_t heads = 0;  // of chunk `lane` of the wave
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const int i = base + u * kWave;
    if (live[u]) keys_out[i] = x[u][0], places_out[i] = x[u][1];
    const uint64_t m = ballot64(live[u] && x[u][0] != (uint32_t)in.n_rows && (i == 0 || lds->pair[i - 1][0] != x[u][0]));
    if (lane_id() == 2 * u) heads = (uint32_t)__popcll(m & 0xFFFFFFFFull);
    if (lane_id() == 2 * u + 1) heads = (uint32_t)__popcll(m >> 32);
  }
  if (in_tile == nullptr) return;
  const uint32_t upto = wave_incl_scan(heads);
  if (lane_id() == kWave - 1) lds->sums[wave_in_block()] = upto;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int w = 0; w < kSortWaves; ++w) {
    before += w < wave_in_block() ? lds->sums[w] : 0;
    all += lds->sums[w];
  }
  const int chunk = wave_in_block() * (2 * kKeysPerThread) + lane_id();
  if (lane_id() < 2 * kKeysPerThread && chunk * 32 < n) in_tile[chunk] = before + upto - heads;
  if (threadIdx.x == 0) *total = all;
}

// n <= kFewTokens: a token's place is the number of those in front of it, one comparison each; 512 of them, ids of 19 bits: 6 us, three
// passes by digits 22.
constexpr int kFewTokens = 512;
__global__ __launch_bounds__(kFewTokens) void k_sort_few(SortInput in, int n, uint32_t* __restrict__ keys_out, uint32_t* __restrict__ places_out,
                                                         uint32_t* __restrict__ in_tile, uint32_t* __restrict__ total, int32_t* __restrict__ bad,
                                                         Zeros zeros) {
  if (blockIdx.x != 0) return zeros.write(blockIdx.x - 1, gridDim.x - 1);
  __shared__ __attribute__((aligned(16))) uint32_t key[kFewTokens];
  __shared__ uint32_t sorted[kFewTokens];
  __shared__ uint32_t heads[2 * kFewTokens / kWave];
  const int i = threadIdx.x;
  bool wrong = false;
  const uint32_t mine = i < n ? in.at(i, &wrong)[0] : 0xFFFFFFFFu;  // (larger than any key)
  if (wrong) atomicOr(bad, 1);
  key[i] = mine;
  __syncthreads();
  uint32_t rank = 0;
#pragma unroll 4
  for (int j = 0; j < n; j += 4) {
    const u32x4 k = *reinterpret_cast<const u32x4*>(key + j);
#pragma unroll
    for (int e = 0; e < 4; ++e) rank += k[e] < mine || (k[e] == mine && j + e < i) ? 1u : 0u;
  }
  if (i < n) {
    sorted[rank] = mine;
    keys_out[rank] = mine;
    places_out[rank] = (uint32_t)i;
  }
  if (in_tile == nullptr) return;
  __syncthreads();
  const uint64_t m = ballot64(i < n && sorted[i] != (uint32_t)in.n_rows && (i == 0 || sorted[i - 1] != sorted[i]));
  if ((lane_id() & 31) == 0) heads[i / 32] = (uint32_t)__popcll(lane_id() == 0 ? m & 0xFFFFFFFFull : m >> 32);
  __syncthreads();
  if (i > 2 * kFewTokens / kWave) return;
  uint32_t before = 0;
  for (int c = 0; c < i; ++c) before += heads[c];
  if (i * 32 < n) in_tile[i] = before;
  if (i == 2 * kFewTokens / kWave) *total = before;
}

// ---- the rows' sums ----------------------------------------------------------------------------------------------------
// The sorted tokens are cut into chunks of kChunk, each summed by a group of lanes that holds a row's columns (E of them each; wider
// rows in column tiles, blockIdx.y).  What begins and ends inside a chunk is written as it is; a row whose tokens run over a chunk's
// end leaves a partial sum per chunk: in slot 1 of the chunk it begins in, in slot 0 of the others.  A row with very many tokens fills
// whole spans of 32 and of 1,024 chunks, whose partial sums k_embed_spans adds up ahead, and k_embed_join adds a row's chunks and
// spans in their order.  No order depends on time: the same input gives the same bits.
// 1,019,311 tokens of 128 elements of bf16, 572,596 rows of fp32: the sums 112 us, 261 MB read and 304 written at 5.0 TB/s; rows' numbers
// (k_embed_heads) 8, spans 6, join 18 us.  A scaled dense gradient of 65,537 tokens of 75 elements is seven launches of 5 to 14 us.
constexpr int kChunk = 32;
constexpr int kAhead = 8;      // rows in flight per group
constexpr int kSpan = 32;      // chunks
constexpr int kSpan2 = 1024;
constexpr int kHeadTile = 4096;                      // tokens
constexpr int kTileChunks = kHeadTile / kChunk;
constexpr int64_t kMaxTokens = (int64_t)1 << 30;     // of a gradient: its launches stay below 2^32 threads
constexpr int32_t kMaxDim = 65535 * 4 * kWave;       // ... and have as many column tiles at most as a grid has rows

struct ReduceShape {
  int64_t n_ids, n_chunks;
  int32_t dim;
  uint32_t n_rows;
  int lanes, lanes_log2;  // per row
};

// The rows form: where a chunk's rows go.  A tile's chunks hold the rows that begin in the tile's chunks in front of them, and a tile those
// in the tiles in front (null: there is one tile).
struct RowPlaces {
  const uint32_t *in_tile, *tile;
  const uint32_t* total;
  __device__ __forceinline__ bool used() const { return in_tile != nullptr; }
  __device__ __forceinline__ int64_t first(int64_t chunk) const {
    return (int64_t)in_tile[chunk] + (tile != nullptr ? (int64_t)tile[chunk / kTileChunks] : 0);
  }
};

__global__ __launch_bounds__(kBlock) void k_embed_heads(const uint32_t* __restrict__ keys, int64_t n, uint32_t n_rows, uint32_t* __restrict__ in_tile,
                                                        uint32_t* __restrict__ tile_sum) {
  static_assert(kChunk == 32 && kTileChunks == 2 * kWave, "half a wave has a chunk; a wave scans the tile's chunks, two a lane");
  __shared__ uint32_t heads[kTileChunks];
  const int64_t base = (int64_t)blockIdx.x * kHeadTile;
#pragma unroll 4
  for (int u = 0; u < kHeadTile / kBlock; ++u) {
    const int at = u * kBlock + threadIdx.x;
    const int64_t i = base + at;
    const uint32_t k = i < n ? keys[i] : n_rows, before = i < n && i > 0 ? keys[i - 1] : n_rows;
    const uint64_t m = ballot64(k != n_rows && k != before);
    if ((lane_id() & 31) == 0) heads[at / kChunk] = (uint32_t)__popcll(lane_id() == 0 ? m & 0xFFFFFFFFull : m >> 32);
  }
  __syncthreads();
  if (threadIdx.x >= kWave) return;
  const uint32_t a = heads[2 * threadIdx.x], b = heads[2 * threadIdx.x + 1], upto = wave_incl_scan(a + b);
  const int64_t chunk = base / kChunk + 2 * threadIdx.x, chunks = (n + kChunk - 1) / kChunk;
  if (chunk < chunks) in_tile[chunk] = upto - a - b;
  if (chunk + 1 < chunks) in_tile[chunk + 1] = upto - b;
  if (threadIdx.x == kWave - 1) tile_sum[blockIdx.x] = upto;
}

template <int TO, int E>
__device__ __forceinline__ void put_row(char* __restrict__ out, int64_t row, int32_t dim, int32_t col, const float (&acc)[E]) {
  Pack<TO, E> y;
  y.set(acc);
  y.store_nt(out + (row * dim + col) * (int64_t)sizeof(typename Element<TO>::M));
}

// a lane's columns of a row; false for a lane that has none
template <int E>
__device__ __forceinline__ bool lane_columns(const ReduceShape& sh, int32_t* col) {
  const int32_t item = (int32_t)blockIdx.y * sh.lanes + (threadIdx.x & (sh.lanes - 1));
  *col = item * E < sh.dim - E ? item * E : sh.dim - E;
  return (int64_t)item * E < sh.dim;
}

template <int TI, int TO, int E>
__global__ __launch_bounds__(kBlock) void k_embed_sum(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places, ReduceShape sh,
                                                      const char* __restrict__ dout, const float* __restrict__ scale, float alpha,
                                                      RowPlaces rp, int32_t* __restrict__ rows_out, int32_t* __restrict__ count,
                                                      char* __restrict__ out, float* __restrict__ part) {
  typedef Pack<TI, E> In;
  const int64_t chunk = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2;
  const int64_t beg = chunk * kChunk, end = beg + kChunk < sh.n_ids ? beg + kChunk : sh.n_ids;
  int32_t col;
  const bool mine = lane_columns<E>(sh, &col), names = col == 0 && rp.used();  // (dim >= E: a column 0 is a row's first item)
  if (rp.used() && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *count = (int32_t)*rp.total;
  if (beg >= end || !mine) return;
  uint32_t cur = keys[beg];
  if (cur == sh.n_rows) return;
  bool begun = beg == 0 || keys[beg - 1] != cur;  // the current row's first token is in this chunk
  int64_t row = rp.used() ? rp.first(chunk) + (begun ? 0 : -1) : (int64_t)cur;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (begun && names) rows_out[row] = (int32_t)cur;
  bool live = true;
  uint32_t next_key[kAhead], next_place[kAhead];  // (known a round ahead: a round then waits for its rows alone)
  const auto look_ahead = [&](int64_t i) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t j = i + u < end ? i + u : end - 1;
      next_place[u] = places[j];
      next_key[u] = keys[j];
    }
  };
  look_ahead(beg);
  for (int64_t i = beg; i < end && live; i += kAhead) {
    uint32_t key[kAhead];
    In x[kAhead];
    float s[kAhead];
    if (scale != nullptr) {  // (one branch for all of them: behind a branch each, each would be waited for by itself)
#pragma unroll
      for (int u = 0; u < kAhead; ++u) s[u] = scale[next_place[u]];
    } else {
#pragma unroll
      for (int u = 0; u < kAhead; ++u) s[u] = 1.f;
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      key[u] = next_key[u];
      x[u] = In::load(dout + ((int64_t)next_place[u] * sh.dim + col) * (int64_t)sizeof(typename In::M));
    }
    if (i + kAhead < end) look_ahead(i + kAhead);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (!live || i + u >= end) continue;
      if (key[u] != cur) {
        if (begun) put_row<TO, E>(out, row, sh.dim, col, acc);
        else store_elements<COOP_F32, E>(part + (2 * chunk * sh.dim + col), acc);
        cur = key[u];
        live = cur != sh.n_rows;
        begun = true;
        row = rp.used() ? row + 1 : (int64_t)cur;
        if (live && names) rows_out[row] = (int32_t)cur;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      if (live) {
        float f[E];
        x[u].get(f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(f[e], s[u] * alpha, acc[e]);
      }
    }
  }
  if (!live) return;
  const bool over = end < sh.n_ids && keys[end] == cur;
  if (begun && !over) put_row<TO, E>(out, row, sh.dim, col, acc);
  else store_elements<COOP_F32, E>(part + ((2 * chunk + (begun ? 1 : 0)) * sh.dim + col), acc);
}

// acc += the partial sums from, from + 1, .. to - 1, `stride` floats apart, in their order
template <int E>
__device__ __forceinline__ void add_parts(const float* p, int64_t stride, int64_t from, int64_t to, float (&acc)[E]) {
  for (int64_t c = from; c < to; c += kAhead) {
    float f[kAhead][E];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) load_elements<COOP_F32, E>(p + (c + u < to ? c + u : to - 1) * stride, f[u]);
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
      if (c + u < to)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += f[u][e];
  }
}

// One row's tokens, begun earlier, fill chunks [c, c + n) (all of them there)
__device__ __forceinline__ bool filled(const uint32_t* keys, const ReduceShape& sh, int64_t c, int n) {
  const int64_t beg = c * kChunk, end = beg + (int64_t)n * kChunk;
  if (beg == 0 || end > sh.n_ids) return false;
  const uint32_t k = keys[beg];
  return k != sh.n_rows && keys[beg - 1] == k && keys[end - 1] == k;
}

// spans[s]: the sum of the partial sums of 32 chunks, by a group of lanes; spans2[t] of 1,024, by a block (the first n_span2 of them)
template <int E>
__global__ __launch_bounds__(kBlock) void k_embed_spans(const uint32_t* __restrict__ keys, ReduceShape sh, const float* __restrict__ part,
                                                        float* __restrict__ spans, float* __restrict__ spans2, int64_t n_span2) {
  __shared__ float lds[E * kBlock];
  int32_t col;
  const bool mine = lane_columns<E>(sh, &col);
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (blockIdx.x < n_span2) {
    const int64_t c = (int64_t)blockIdx.x * kSpan2;
    if (!filled(keys, sh, c, kSpan2)) return;  // (the whole block)
    const int groups = kBlock >> sh.lanes_log2, g = threadIdx.x >> sh.lanes_log2, each = kSpan2 / groups;
    if (mine) add_parts<E>(part + col, 2 * (int64_t)sh.dim, c + g * each, c + (g + 1) * each, acc);
#pragma unroll
    for (int e = 0; e < E; ++e) lds[e * kBlock + threadIdx.x] = acc[e];
    __syncthreads();
    if (g != 0 || !mine) return;
    for (int o = 1; o < groups; ++o)
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += lds[e * kBlock + (o << sh.lanes_log2) + threadIdx.x];
    store_elements<COOP_F32, E>(spans2 + (int64_t)blockIdx.x * sh.dim + col, acc);
    return;
  }
  const int64_t s = (((int64_t)blockIdx.x - n_span2) * kBlock + threadIdx.x) >> sh.lanes_log2;
  if (s * kSpan >= sh.n_chunks || !mine || !filled(keys, sh, s * kSpan, kSpan)) return;
  add_parts<E>(part + col, 2 * (int64_t)sh.dim, s * kSpan, (s + 1) * kSpan, acc);
  store_elements<COOP_F32, E>(spans + s * sh.dim + col, acc);
}

// A group of lanes per chunk: if a row begins in the chunk and runs over its end, the partial sums of all its chunks.
template <int TO, int E>
__global__ __launch_bounds__(kBlock) void k_embed_join(const uint32_t* __restrict__ keys, ReduceShape sh, RowPlaces rp,
                                                       const float* __restrict__ part, const float* __restrict__ spans,
                                                       const float* __restrict__ spans2, char* __restrict__ out) {
  const int64_t chunk = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2;
  int32_t col;
  if (!lane_columns<E>(sh, &col) || chunk + 1 >= sh.n_chunks) return;
  const int64_t beg = chunk * kChunk, next = beg + kChunk;
  const uint32_t cur = keys[next];
  if (cur == sh.n_rows || keys[next - 1] != cur || (keys[beg] == cur && beg != 0 && keys[beg - 1] == cur)) return;
  // the first chunk that does not begin with this row: doubling steps, then halving
  int64_t in = chunk + 1, out_of = sh.n_chunks;
  for (int64_t step = 1; in + step < out_of; step *= 2) {
    if (keys[(in + step) * kChunk] != cur) {
      out_of = in + step;
      break;
    }
    in += step;
  }
  while (out_of - in > 1) {
    const int64_t mid = (in + out_of) / 2;
    if (keys[mid * kChunk] == cur) in = mid;
    else out_of = mid;
  }
  float acc[E];
  const float* slot0 = part + col;
  const int64_t stride = 2 * (int64_t)sh.dim;
  load_elements<COOP_F32, E>(part + ((2 * chunk + 1) * sh.dim + col), acc);
  // what is whole of the spans; the last chunk may hold other rows as well, and then is none of a span's
  const int64_t whole = out_of * kChunk <= sh.n_ids && keys[out_of * kChunk - 1] == cur ? out_of : out_of - 1;
  int64_t c = chunk + 1;
  const auto up_to = [](int64_t x, int64_t to) { return (x + to - 1) / to * to; };
  const int64_t s0 = up_to(c, kSpan), s1 = whole / kSpan * kSpan;
  if (spans != nullptr && s0 < s1) {
    add_parts<E>(slot0, stride, c, s0, acc);
    c = s0;
    const int64_t t0 = up_to(s0, kSpan2), t1 = s1 / kSpan2 * kSpan2;
    if (t0 < t1) {
      add_parts<E>(spans + col, sh.dim, c / kSpan, t0 / kSpan, acc);
      add_parts<E>(spans2 + col, sh.dim, t0 / kSpan2, t1 / kSpan2, acc);
      c = t1;
    }
    add_parts<E>(spans + col, sh.dim, c / kSpan, s1 / kSpan, acc);
    c = s1;
  }
  add_parts<E>(slot0, stride, c, out_of, acc);
  put_row<TO, E>(out, rp.used() ? rp.first(chunk + 1) - 1 : (int64_t)cur, sh.dim, col, acc);
}

__global__ void k_embed_none(int32_t* __restrict__ count) { *count = 0; }

// ---- the workspace of a gradient -----------------------------------------------------------------------------------------
struct GradPlan {
  int64_t n, tiles, head_tiles, chunks, n_span, n_span2;
  size_t pairs[2], keys, places, matrix, place, scan, in_tile, tile_sum, tile, part, spans, spans2, bytes;
  GradPlan(int64_t n_ids, int32_t dim) : n(n_ids) {
    tiles = (n + kSortTile - 1) / kSortTile;
    head_tiles = (n + kHeadTile - 1) / kHeadTile;
    chunks = (n + kChunk - 1) / kChunk;
    n_span = chunks / kSpan;
    n_span2 = chunks / kSpan2;
    const int64_t cells = tiles > 1 ? tiles << kDigitBits : 0;
    size_t at = 0;
    auto take = [&](size_t b) { const size_t o = at; at += (b + 255) & ~(size_t)255; return o; };
    for (int i = 0; i < 2; ++i) pairs[i] = take(tiles > 1 ? (size_t)n * 8 : 0);
    keys = take((size_t)n * 4);
    places = take((size_t)n * 4);
    matrix = take((size_t)(cells + 1) * 4);
    place = take(tiles > kOwnTiles ? (size_t)(cells + 1) * 4 : 0);
    in_tile = take((size_t)chunks * 4);
    tile_sum = take((size_t)(head_tiles + 1) * 4);
    tile = take((size_t)(head_tiles + 1) * 4);
    const size_t t1 = scan_tmp_bytes(cells), t2 = scan_tmp_bytes(head_tiles);
    scan = take(t1 > t2 ? t1 : t2);
    part = take((size_t)chunks * 2 * (size_t)dim * 4);
    spans = take((size_t)n_span * (size_t)dim * 4);
    spans2 = take((size_t)n_span2 * (size_t)dim * 4);
    bytes = at + 256;
  }
};

template <int TI, int TO, int E>
void launch_reduce(const GradPlan& plan, char* ws, const uint32_t* keys, const uint32_t* places, const RowPlaces& rp, int64_t n_rows,
                   int32_t dim, const void* dout, const float* scale, float alpha, int32_t* rows_out, int32_t* count, void* grad, hipStream_t s) {
  const int32_t items = (dim + E - 1) / E;
  ReduceShape sh{plan.n, plan.chunks, dim, (uint32_t)n_rows, 1, 0};
  while (sh.lanes < items && sh.lanes < kWave) sh.lanes *= 2, ++sh.lanes_log2;
  const unsigned col_tiles = (unsigned)((items + sh.lanes - 1) / sh.lanes);
  const auto blocks = [&](int64_t groups) { return (groups * sh.lanes + kBlock - 1) / kBlock; };
  const dim3 grid((unsigned)blocks(plan.chunks), col_tiles);
  float* part = (float*)(ws + plan.part);
  float* spans = plan.n_span > 0 ? (float*)(ws + plan.spans) : nullptr;
  float* spans2 = (float*)(ws + plan.spans2);
  COOP_LAUNCH(K_EMBED_SUM, (k_embed_sum<TI, TO, E>), grid, dim3(kBlock), 0, s, keys, places, sh, (const char*)dout, scale, alpha, rp,
              rows_out, count, (char*)grad, part);
  if (plan.chunks == 1) return;
  if (spans != nullptr)
    COOP_LAUNCH(K_EMBED_SPANS, k_embed_spans<E>, dim3((unsigned)(plan.n_span2 + blocks(plan.n_span)), col_tiles), dim3(kBlock), 0, s, keys, sh,
                (const float*)part, spans, spans2, plan.n_span2);
  COOP_LAUNCH(K_EMBED_JOIN, (k_embed_join<TO, E>), grid, dim3(kBlock), 0, s, keys, sh, rp, (const float*)part, (const float*)spans,
              (const float*)spans2, (char*)grad);
}

// the ids' tokens, sorted, into the workspace's keys and places, and `zeros` in equal parts by all launches
template <bool OWN>
void sort_passes(const GradPlan& plan, char* ws, SortInput in, int bits, int32_t* bad, const Zeros& zeros, hipStream_t s) {
  uint32_t* matrix = (uint32_t*)(ws + plan.matrix);
  uint32_t* counts = OWN ? matrix : (uint32_t*)(ws + plan.place);
  const dim3 block(kSortBlock);
  const uint32_t tiles = (uint32_t)plan.tiles;
  const int launches = (bits + kDigitBits - 1) / kDigitBits * 2;
  int to = 0, launch = 0;
  for (int shift = 0; shift < bits; shift += kDigitBits, to ^= 1) {
    const bool last = shift + kDigitBits >= bits;
    u32x2* pairs = (u32x2*)(ws + plan.pairs[to]);
    const Zeros first = zeros.part(launch, launches), second = zeros.part(launch + 1, launches);
    launch += 2;
    COOP_LAUNCH(K_SORT_COUNT, k_sort_count<OWN>, dim3(tiles + first.blocks(kSortBlock)), block, 0, s, in, plan.n, shift, matrix, tiles, bad, first);
    if (!OWN) scan_u32_to_u32(matrix, plan.tiles << kDigitBits, counts, ws + plan.scan, s);
    COOP_LAUNCH(K_SORT_PLACE, k_sort_place<OWN>, dim3(tiles + second.blocks(kSortBlock)), block, sizeof(SortLds), s, in, plan.n, shift,
                (const uint32_t*)counts, tiles, pairs, last ? (uint32_t*)(ws + plan.keys) : nullptr, last ? (uint32_t*)(ws + plan.places) : nullptr, second);
    in.ids = nullptr;
    in.pairs = pairs;
  }
}

template <typename K>
bool allow_sort(K kernel) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(SortLds)) == hipSuccess;
}

int grad_launch(const void* dout, int dtype, const int32_t* ids, int64_t n, const float* scale, float alpha, int32_t pad, int64_t n_rows,
                int32_t dim, void* grad, int grad_dtype, int32_t* rows_out, int32_t* count, bool rows_form, void* workspace, size_t ws_bytes,
                hipStream_t s) {
  if (!known_dtype(dtype) || !known_dtype(grad_dtype)) return COOP_E_ARG;
  if (n < 0 || n > kMaxTokens || n_rows < 0 || n_rows >= ((int64_t)1 << 31) || dim < 1 || dim > kMaxDim) return COOP_E_ARG;
  if (rows_form && !count) return COOP_E_NULL;
  if (n > 0 && (!dout || !ids || !workspace)) return COOP_E_NULL;
  if ((rows_form ? (n < n_rows ? n : n_rows) : n_rows) > 0 && (!grad || (rows_form && !rows_out))) return COOP_E_NULL;
  if (!aligned_for(dout, dtype) || !aligned_for(grad, grad_dtype)) return COOP_E_ARG;
  const GradPlan plan(n, dim);
  if (n > 0 && (ws_bytes < plan.bytes || ((uintptr_t)workspace & 255) != 0)) return COOP_E_ARG;
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  const int64_t dense = rows_form ? 0 : n_rows * dim * element_bytes(grad_dtype);
  if (n == 0) {
    clear_bytes(grad, dense, s);
    if (rows_form) COOP_LAUNCH(K_EMBED_HEADS, k_embed_none, dim3(1), dim3(1), 0, s, count);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
  }
  char* ws = (char*)workspace;
  int bits = 1;
  while ((n_rows >> bits) != 0) ++bits;  // (the keys are 0 .. n_rows)
  const SortInput in{ids, nullptr, n_rows, pad};
  uint32_t* keys = (uint32_t*)(ws + plan.keys);
  uint32_t* places = (uint32_t*)(ws + plan.places);
  const Zeros zeros = zeros_of(grad, dense);
  if (n <= kFewTokens) {
    COOP_LAUNCH(K_SORT_PLACE, k_sort_few, dim3(1 + zeros.blocks(kFewTokens)), dim3(kFewTokens), 0, s, in, (int)n, keys, places,
                rows_form ? (uint32_t*)(ws + plan.in_tile) : nullptr, (uint32_t*)(ws + plan.tile_sum), bad, zeros);
  } else if (plan.tiles == 1) {
    if (!allow_sort(k_sort_small)) return COOP_E_HIP;
    COOP_LAUNCH(K_SORT_PLACE, k_sort_small, dim3(1 + zeros.blocks(kSortBlock)), dim3(kSortBlock), sizeof(SortLds), s, in, (int)n, bits, keys, places,
                rows_form ? (uint32_t*)(ws + plan.in_tile) : nullptr, (uint32_t*)(ws + plan.tile_sum), bad, zeros);
  } else if (plan.tiles <= kOwnTiles) {
    if (!allow_sort(k_sort_place<true>)) return COOP_E_HIP;
    sort_passes<true>(plan, ws, in, bits, bad, zeros, s);
  } else {
    if (!allow_sort(k_sort_place<false>)) return COOP_E_HIP;
    sort_passes<false>(plan, ws, in, bits, bad, zeros, s);
  }
  RowPlaces rp{nullptr, nullptr, nullptr};
  if (rows_form) {
    uint32_t* tile_sum = (uint32_t*)(ws + plan.tile_sum);
    uint32_t* tile = (uint32_t*)(ws + plan.tile);
    const bool one = plan.tiles == 1;  // (the sort has left it)
    if (!one) COOP_LAUNCH(K_EMBED_HEADS, k_embed_heads, dim3((unsigned)plan.head_tiles), dim3(kBlock), 0, s, keys, n, (uint32_t)n_rows,
                (uint32_t*)(ws + plan.in_tile), tile_sum);
    if (!one) scan_u32_to_u32(tile_sum, plan.head_tiles, tile, ws + plan.scan, s);
    rp = RowPlaces{(const uint32_t*)(ws + plan.in_tile), one ? nullptr : tile, one ? tile_sum : tile + plan.head_tiles};
  }
  with_dtype(dtype, [&](auto ti) {
    with_dtype(grad_dtype, [&](auto to_) {
      constexpr int TI = decltype(ti)::value, TO = decltype(to_)::value, E = TI == COOP_F32 || TO == COOP_F32 ? 4 : 8;
      const auto go = [&](auto e) {
        launch_reduce<TI, TO, decltype(e)::value>(plan, ws, keys, places, rp, n_rows, dim, dout, scale, alpha, rows_out, count, grad, s);
      };
      // (16 bytes a lane of the gradient's row, or of the tokens'; rows of fewer columns go one by one)
      if (dim >= E) go(std::integral_constant<int, E>());
      else go(std::integral_constant<int, 1>());
    });
  });
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

}  // namespace
}  // namespace coop

using namespace coop;

extern "C" int coop_embed(const void* table, int64_t n_rows, int32_t dim, int dtype, const int32_t* ids, int64_t n_ids, const float* scale,
                          float alpha, int32_t pad, void* out, int out_dtype, void* stream) {
  if (!known_dtype(dtype) || !known_dtype(out_dtype)) return COOP_E_ARG;
  if (dim < 1 || n_rows < 0 || n_rows >= ((int64_t)1 << 31) || n_ids < 0) return COOP_E_ARG;
  if (n_ids == 0) return COOP_OK;
  if (n_rows == 0) return COOP_E_ARG;
  if (!table || !ids || !out) return COOP_E_NULL;
  if (!aligned_for(table, dtype) || !aligned_for(out, out_dtype)) return COOP_E_ARG;
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  hipStream_t s = (hipStream_t)stream;
  with_dtype(dtype, [&](auto ti) {
    with_dtype(out_dtype, [&](auto to) {
      constexpr int TI = decltype(ti)::value, TO = decltype(to)::value, E = TI == COOP_F32 || TO == COOP_F32 ? 4 : 8;
      const auto go = [&](auto e) {
        constexpr int N = decltype(e)::value;
        const uint32_t vecs = (uint32_t)(((int64_t)dim + N - 1) / N);
        constexpr int64_t per_block = kBlock * kUnroll;
        const int64_t most = kSliceBlocks * per_block / (int64_t)vecs;  // ids of a launch of fewer than 2^32 threads
        for (int64_t i = 0; i < n_ids; i += most) {
          const int64_t n = n_ids - i < most ? n_ids - i : most;
          const EmbedShape sh{n_rows, n, dim, pad, vecs, (uint32_t)((((uint64_t)1 << 32) + vecs - 1) / vecs)};
          COOP_LAUNCH(K_EMBED, (k_embed<TI, TO, N>), dim3((unsigned)((n * (int64_t)vecs + per_block - 1) / per_block)), dim3(kBlock), 0, s,
                      (const char*)table, sh, ids + i, scale != nullptr ? scale + i : nullptr, alpha,
                      (char*)out + i * dim * element_bytes(out_dtype), bad);
        }
      };
      if (dim >= E) go(std::integral_constant<int, E>());
      else go(std::integral_constant<int, 1>());
    });
  });
  return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
}

extern "C" size_t coop_embed_grad_workspace_bytes(int64_t n_ids, int32_t dim) {
  if (n_ids < 0 || n_ids > kMaxTokens || dim < 1 || dim > kMaxDim) return 0;
  return GradPlan(n_ids, dim).bytes;
}

extern "C" int coop_embed_grad(const void* dout, int dtype, const int32_t* ids, int64_t n_ids, const float* scale, float alpha, int32_t pad,
                               int64_t n_rows, int32_t dim, void* grad, int grad_dtype, void* workspace, size_t workspace_bytes, void* stream) {
  return grad_launch(dout, dtype, ids, n_ids, scale, alpha, pad, n_rows, dim, grad, grad_dtype, nullptr, nullptr, false, workspace,
                     workspace_bytes, (hipStream_t)stream);
}

extern "C" int coop_embed_grad_rows(const void* dout, int dtype, const int32_t* ids, int64_t n_ids, const float* scale, float alpha,
                                    int32_t pad, int64_t n_rows, int32_t dim, int32_t* rows_out, void* grad, int grad_dtype,
                                    int32_t* count_out, void* workspace, size_t workspace_bytes, void* stream) {
  return grad_launch(dout, dtype, ids, n_ids, scale, alpha, pad, n_rows, dim, grad, grad_dtype, rows_out, count_out, true, workspace,
                     workspace_bytes, (hipStream_t)stream);
}
