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
constexpr int kUnroll = 4;

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
    if (!ok[u] && id[u] != sh.pad && col[u] == 0) atomicOr(bad, 1);
  }
}

// ---- the tokens in the order of their ids ------------------------------------------------------------------------------
// A stable radix sort of (id, place), least significant digit first: per pass a count of every tile's digits, the exclusive scan of
// the counts in the order (digit, tile), and the placement.  A place without a row has the key n_rows and comes last.
constexpr int kDigitBits = 8;
constexpr int kDigits = 1 << kDigitBits;
constexpr int kKeysPerThread = 16;
constexpr int kSortTile = kBlock * kKeysPerThread;

struct SortInput {  // the first pass reads the ids, the others what the pass before has left
  const int32_t* ids;
  const uint32_t *keys, *places;
  int64_t n_rows;
  int32_t pad;
  __device__ __forceinline__ uint32_t key(int64_t i) const {
    if (ids == nullptr) return keys[i];
    const int32_t id = ids[i];
    return id != pad && (uint64_t)(int64_t)id < (uint64_t)n_rows ? (uint32_t)id : (uint32_t)n_rows;
  }
  __device__ __forceinline__ uint32_t place(int64_t i) const { return ids == nullptr ? places[i] : (uint32_t)i; }
};

__global__ __launch_bounds__(kBlock) void k_sort_count(SortInput in, int64_t n, int shift, uint32_t* __restrict__ matrix, uint32_t tiles,
                                                       int32_t* __restrict__ bad) {
  __shared__ uint32_t cnt[kDigits];
  cnt[threadIdx.x] = 0;
  __syncthreads();
  const int64_t base = (int64_t)blockIdx.x * kSortTile;
  bool wrong = false;
#pragma unroll 4
  for (int u = 0; u < kKeysPerThread; ++u) {
    const int64_t i = base + u * kBlock + threadIdx.x;
    if (i < n) {
      const uint32_t k = in.key(i);
      atomicAdd(&cnt[k >> shift & (kDigits - 1)], 1u);
      wrong |= in.ids != nullptr && k == (uint32_t)in.n_rows && in.ids[i] != in.pad;
    }
  }
  if (wrong) atomicOr(bad, 1);
  __syncthreads();
  matrix[(size_t)threadIdx.x * tiles + blockIdx.x] = cnt[threadIdx.x];
}

// the lanes of this wave whose digit is the same
__device__ __forceinline__ uint64_t same_digit(uint32_t digit, uint64_t live) {
  uint64_t m = live;
#pragma unroll
  for (int b = 0; b < kDigitBits; ++b) {
    const uint64_t set = ballot64(digit >> b & 1);
    m &= digit >> b & 1 ? set : ~set;
  }
  return m;
}

__global__ __launch_bounds__(kBlock) void k_sort_place(SortInput in, int64_t n, int shift, const uint32_t* __restrict__ first, uint32_t tiles,
                                                       uint32_t* __restrict__ keys_out, uint32_t* __restrict__ places_out) {
  static_assert(kDigits == kBlock, "a thread has a digit");
  __shared__ uint32_t cnt[kWavesPerBlock][kDigits];
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) cnt[w][threadIdx.x] = 0;
  __syncthreads();
  const int wave = uniform_wave_in_block();
  const int64_t base = (int64_t)blockIdx.x * kSortTile + wave * (kKeysPerThread * kWave) + lane_id();
  uint32_t key[kKeysPerThread], place[kKeysPerThread], rank[kKeysPerThread];
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const int64_t i = base + u * kWave;
    key[u] = i < n ? in.key(i) : 0u;
    place[u] = i < n ? in.place(i) : 0u;
  }
  // a wave's keys in order, 64 at a time: how many of the same digit are in front
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    const bool live = base + u * kWave < n;
    const uint32_t d = key[u] >> shift & (kDigits - 1);
    const uint64_t same = same_digit(d, ballot64(live));
    const uint32_t before = lanes_below(same);
    const uint32_t ran = live ? cnt[wave][d] : 0u;
    rank[u] = ran + before;
    __builtin_amdgcn_wave_barrier();
    if (live && before == 0) cnt[wave][d] = ran + (uint32_t)__popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
  uint32_t at = first[(size_t)threadIdx.x * tiles + blockIdx.x];
#pragma unroll
  for (int w = 0; w < kWavesPerBlock; ++w) {
    const uint32_t c = cnt[w][threadIdx.x];
    cnt[w][threadIdx.x] = at;
    at += c;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < kKeysPerThread; ++u) {
    if (base + u * kWave >= n) continue;
    const uint32_t to = cnt[wave][key[u] >> shift & (kDigits - 1)] + rank[u];
    keys_out[to] = key[u];
    places_out[to] = place[u];
  }
}

// ---- the rows' sums ----------------------------------------------------------------------------------------------------
// The sorted tokens are cut into chunks of kChunk, each summed by a group of lanes that holds a row's columns (E of them each; wider
// rows in column tiles, blockIdx.y).  What begins and ends inside a chunk is written as it is; a row whose tokens run over a chunk's
// end leaves a partial sum per chunk (slot 1 of the chunk it begins in, slot 0 of the others), which k_embed_join adds up in order.
// No order depends on time: the same input gives the same bits.
constexpr int kChunk = 32;
constexpr int kAhead = 8;  // rows in flight per group
constexpr int64_t kMaxTokens = (int64_t)1 << 30;  // of a gradient: its launches stay below 2^32 threads

struct ReduceShape {
  int64_t n_ids;
  int32_t dim;
  uint32_t n_rows;
  int lanes, lanes_log2;  // per row
};

// heads: the tokens of each chunk that are the first with their id
__global__ __launch_bounds__(kBlock) void k_embed_heads(const uint32_t* __restrict__ keys, int64_t n, uint32_t n_rows, uint32_t* __restrict__ heads,
                                                        int64_t n_chunks) {
  const int64_t i = (int64_t)blockIdx.x * kBlock + threadIdx.x;
  const uint32_t k = i < n ? keys[i] : n_rows;
  const bool head = k != n_rows && (i == 0 || keys[i - 1] != k);
  const uint64_t m = ballot64(head);
  static_assert(kChunk == 32, "half a wave has a chunk");
  if ((lane_id() & 31) == 0 && i / kChunk < n_chunks) heads[i / kChunk] = (uint32_t)__popcll(lane_id() == 0 ? m & 0xFFFFFFFFull : m >> 32);
}

template <int TO, int E>
__device__ __forceinline__ void put_row(char* __restrict__ out, int64_t row, int32_t dim, int32_t col, const float (&acc)[E]) {
  Pack<TO, E> y;
  y.set(acc);
  y.store_nt(out + (row * dim + col) * (int64_t)sizeof(typename Pack<TO, E>::M));
}

// `first`: the rows in front of each chunk's first head (the rows form), or null: a row's place is its id
template <int TI, int TO, int E>
__global__ __launch_bounds__(kBlock) void k_embed_sum(const uint32_t* __restrict__ keys, const uint32_t* __restrict__ places, ReduceShape sh,
                                                      const char* __restrict__ dout, const float* __restrict__ scale, float alpha,
                                                      const uint32_t* __restrict__ first, int32_t* __restrict__ rows_out,
                                                      char* __restrict__ out, float* __restrict__ part) {
  typedef Pack<TI, E> In;
  const int64_t chunk = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2;
  const int lane = threadIdx.x & (sh.lanes - 1);
  const int64_t beg = chunk * kChunk, end = beg + kChunk < sh.n_ids ? beg + kChunk : sh.n_ids;
  const int32_t item = (int32_t)blockIdx.y * sh.lanes + lane;
  if (beg >= end || (int64_t)item * E >= sh.dim) return;
  const int32_t col = item * E < sh.dim - E ? item * E : sh.dim - E;
  uint32_t cur = keys[beg];
  if (cur == sh.n_rows) return;
  bool begun = beg == 0 || keys[beg - 1] != cur;  // the current row's first token is in this chunk
  int64_t row = first != nullptr ? (int64_t)first[chunk] + (begun ? 0 : -1) : (int64_t)cur;
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  if (begun && first != nullptr && item == 0) rows_out[row] = (int32_t)cur;
  bool live = true;
  for (int64_t i = beg; i < end && live; i += kAhead) {
    uint32_t key[kAhead];
    In x[kAhead];
    float s[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int64_t j = i + u < end ? i + u : end - 1;
      const uint32_t place = places[j];
      key[u] = i + u < end ? keys[j] : sh.n_rows;
      s[u] = scale != nullptr ? scale[place] * alpha : alpha;
      x[u] = In::load(dout + ((int64_t)place * sh.dim + col) * (int64_t)sizeof(typename In::M));
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (!live || i + u >= end) continue;
      if (key[u] != cur) {
        if (begun) put_row<TO, E>(out, row, sh.dim, col, acc);
        else store_elements<COOP_F32, E>(part + (2 * chunk * sh.dim + col), acc);
        cur = key[u];
        live = cur != sh.n_rows;
        begun = true;
        row = first != nullptr ? row + 1 : (int64_t)cur;
        if (live && first != nullptr && item == 0) rows_out[row] = (int32_t)cur;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      if (live) {
        float f[E];
        x[u].get(f);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = __builtin_fmaf(f[e], s[u], acc[e]);
      }
    }
  }
  if (!live) return;
  const bool over = end < sh.n_ids && keys[end] == cur;
  if (begun && !over) put_row<TO, E>(out, row, sh.dim, col, acc);
  else store_elements<COOP_F32, E>(part + ((2 * chunk + (begun ? 1 : 0)) * sh.dim + col), acc);
}

// A group of lanes per chunk: if a row begins in the chunk and runs over its end, the partial sums of all its chunks.
template <int TO, int E>
__global__ __launch_bounds__(kBlock) void k_embed_join(const uint32_t* __restrict__ keys, ReduceShape sh, const uint32_t* __restrict__ first,
                                                       int64_t n_chunks, const float* __restrict__ part, char* __restrict__ out) {
  const int64_t chunk = ((int64_t)blockIdx.x * kBlock + threadIdx.x) >> sh.lanes_log2;
  const int lane = threadIdx.x & (sh.lanes - 1);
  const int32_t item = (int32_t)blockIdx.y * sh.lanes + lane;
  if (chunk + 1 >= n_chunks || (int64_t)item * E >= sh.dim) return;
  const int32_t col = item * E < sh.dim - E ? item * E : sh.dim - E;
  const int64_t beg = chunk * kChunk, next = beg + kChunk;
  const uint32_t cur = keys[next];
  if (cur == sh.n_rows || keys[next - 1] != cur || (keys[beg] == cur && beg != 0 && keys[beg - 1] == cur)) return;
  float acc[E];
  load_elements<COOP_F32, E>(part + ((2 * chunk + 1) * sh.dim + col), acc);
  for (int64_t c = chunk + 1; c < n_chunks && keys[c * kChunk] == cur; ++c) {
    float f[E];
    load_elements<COOP_F32, E>(part + (2 * c * sh.dim + col), f);
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] += f[e];
  }
  put_row<TO, E>(out, first != nullptr ? (int64_t)first[chunk + 1] - 1 : (int64_t)cur, sh.dim, col, acc);
}

__global__ void k_embed_count(const uint32_t* __restrict__ total, int32_t* __restrict__ count) {
  *count = total != nullptr ? (int32_t)*total : 0;
}

// ---- the workspace of a gradient -----------------------------------------------------------------------------------------
struct GradPlan {
  int64_t n, tiles, cells, chunks;
  size_t keys[2], places[2], matrix, place, scan, heads, first, part, bytes;
  GradPlan(int64_t n_ids, int32_t dim) : n(n_ids) {
    tiles = (n + kSortTile - 1) / kSortTile;
    cells = tiles * kDigits;
    chunks = (n + kChunk - 1) / kChunk;
    size_t at = 0;
    auto take = [&](size_t b) { const size_t o = at; at += (b + 255) & ~(size_t)255; return o; };
    for (int i = 0; i < 2; ++i) keys[i] = take((size_t)n * 4), places[i] = take((size_t)n * 4);
    matrix = take((size_t)(cells + 1) * 4);
    place = take((size_t)(cells + 1) * 4);
    heads = take((size_t)(chunks + 1) * 4);
    first = take((size_t)(chunks + 1) * 4);
    const size_t t1 = scan_tmp_bytes(cells), t2 = scan_tmp_bytes(chunks);
    scan = take(t1 > t2 ? t1 : t2);
    part = take((size_t)chunks * 2 * (size_t)dim * 4);
    bytes = at + 256;
  }
};

template <int TI, int TO, int E>
void launch_reduce(const GradPlan& plan, char* ws, const uint32_t* keys, const uint32_t* places, const uint32_t* first, int64_t n_rows,
                   int32_t dim, const void* dout, const float* scale, float alpha, int32_t* rows_out, void* grad, hipStream_t s) {
  const int32_t items = (dim + E - 1) / E;
  ReduceShape sh{plan.n, dim, (uint32_t)n_rows, 1, 0};
  while (sh.lanes < items && sh.lanes < kWave) sh.lanes *= 2, ++sh.lanes_log2;
  const dim3 grid((unsigned)((plan.chunks * sh.lanes + kBlock - 1) / kBlock), (unsigned)((items + sh.lanes - 1) / sh.lanes));
  float* part = (float*)(ws + plan.part);
  COOP_LAUNCH(K_EMBED_SUM, (k_embed_sum<TI, TO, E>), grid, dim3(kBlock), 0, s, keys, places, sh, (const char*)dout, scale, alpha, first,
              rows_out, (char*)grad, part);
  if (plan.chunks > 1)
    COOP_LAUNCH(K_EMBED_JOIN, (k_embed_join<TO, E>), grid, dim3(kBlock), 0, s, keys, sh, first, plan.chunks, (const float*)part, (char*)grad);
}

int grad_launch(const void* dout, int dtype, const int32_t* ids, int64_t n, const float* scale, float alpha, int32_t pad, int64_t n_rows,
                int32_t dim, void* grad, int grad_dtype, int32_t* rows_out, int32_t* count, bool rows_form, void* workspace, size_t ws_bytes,
                hipStream_t s) {
  if (!known_dtype(dtype) || !known_dtype(grad_dtype)) return COOP_E_ARG;
  if (n < 0 || n > kMaxTokens || n_rows < 0 || n_rows >= ((int64_t)1 << 31) || dim < 1) return COOP_E_ARG;
  if (rows_form && !count) return COOP_E_NULL;
  if (n > 0 && (!dout || !ids || !workspace)) return COOP_E_NULL;
  if ((rows_form ? (n < n_rows ? n : n_rows) : n_rows) > 0 && (!grad || (rows_form && !rows_out))) return COOP_E_NULL;
  if (!aligned_for(dout, dtype) || !aligned_for(grad, grad_dtype)) return COOP_E_ARG;
  const GradPlan plan(n, dim);
  if (n > 0 && (ws_bytes < plan.bytes || ((uintptr_t)workspace & 255) != 0)) return COOP_E_ARG;
  int32_t* bad = bad_flag();
  if (!bad) return COOP_E_HIP;
  if (!rows_form) clear_bytes(grad, n_rows * dim * element_bytes(grad_dtype), s);
  if (n == 0) {
    if (rows_form) COOP_LAUNCH(K_EMBED_HEADS, k_embed_count, dim3(1), dim3(1), 0, s, (const uint32_t*)nullptr, count);
    return hipGetLastError() == hipSuccess ? COOP_OK : COOP_E_HIP;
  }
  char* ws = (char*)workspace;
  uint32_t* matrix = (uint32_t*)(ws + plan.matrix);
  uint32_t* place = (uint32_t*)(ws + plan.place);
  SortInput in{ids, nullptr, nullptr, n_rows, pad};
  int to = 0;
  for (int shift = 0; shift == 0 || (n_rows >> shift) != 0; shift += kDigitBits) {
    uint32_t* keys_out = (uint32_t*)(ws + plan.keys[to]);
    uint32_t* places_out = (uint32_t*)(ws + plan.places[to]);
    COOP_LAUNCH(K_SORT_COUNT, k_sort_count, dim3((unsigned)plan.tiles), dim3(kBlock), 0, s, in, n, shift, matrix, (uint32_t)plan.tiles, bad);
    scan_u32_to_u32(matrix, plan.cells, place, ws + plan.scan, s);
    COOP_LAUNCH(K_SORT_PLACE, k_sort_place, dim3((unsigned)plan.tiles), dim3(kBlock), 0, s, in, n, shift, (const uint32_t*)place,
                (uint32_t)plan.tiles, keys_out, places_out);
    in = SortInput{nullptr, keys_out, places_out, n_rows, pad};
    to ^= 1;
  }
  const uint32_t* first = nullptr;
  if (rows_form) {
    uint32_t* heads = (uint32_t*)(ws + plan.heads);
    uint32_t* f = (uint32_t*)(ws + plan.first);
    COOP_LAUNCH(K_EMBED_HEADS, k_embed_heads, dim3((unsigned)((n + kBlock - 1) / kBlock)), dim3(kBlock), 0, s, in.keys, n, (uint32_t)n_rows,
                heads, plan.chunks);
    scan_u32_to_u32(heads, plan.chunks, f, ws + plan.scan, s);
    COOP_LAUNCH(K_EMBED_HEADS, k_embed_count, dim3(1), dim3(1), 0, s, (const uint32_t*)(f + plan.chunks), count);
    first = f;
  }
  with_dtype(dtype, [&](auto ti) {
    with_dtype(grad_dtype, [&](auto to_) {
      constexpr int TI = decltype(ti)::value, TO = decltype(to_)::value, E = TI == COOP_F32 ? 4 : 8;
      const auto go = [&](auto e) {
        launch_reduce<TI, TO, decltype(e)::value>(plan, ws, in.keys, in.places, first, n_rows, dim, dout, scale, alpha, rows_out, grad, s);
      };
      // (an accumulator of 8 columns leaves in two 16-byte stores as fp32; rows of fewer columns than a lane holds go one by one)
      constexpr int EO = TO == COOP_F32 ? 4 : E;
      if (dim >= EO) go(std::integral_constant<int, EO>());
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
        const uint32_t vecs = (uint32_t)((dim + N - 1) / N);
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
  if (n_ids < 0 || n_ids > kMaxTokens || dim < 1) return 0;
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
