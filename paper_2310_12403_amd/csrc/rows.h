// Rows that lanes share, for the norms: which columns a lane has, sums over a row, and which rows a block takes.
#pragma once
#include "elements.h"

namespace coop {

// Where a lane's columns are.  A row is cut into packs of E columns, dealt to the lanes in order, K per lane; the last pack is anchored
// at the row's end, and the columns that it shares with the one in front do not count (`own` is the first that does).
template <int E>
struct Columns {
  int32_t at;
  int own;
  bool live;
  __device__ __forceinline__ Columns(int32_t pack, int32_t dim) {
    const int32_t c = pack * E, last = dim - E;
    live = c < dim;
    at = !live ? 0 : c < last ? c : last;
    own = live ? c - at : E;
  }
};

// Sum over the lanes that share a row: WAVES = 1: an aligned group of them in a wave; else the whole block.
template <int WAVES>
__device__ __forceinline__ float row_sum(float v, int lanes, float* lds /* [WAVES] */) {
  if constexpr (WAVES == 1) {
    return group_sum(v, lanes);
  } else {
    v = group_sum(v, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[wave_in_block()] = v;
    __syncthreads();
    float t = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) t += lds[w];
    return t;
  }
}
template <int WAVES>
__device__ __forceinline__ void row_sums(float& a, float& b, int lanes, float* lds /* [2 WAVES] */) {
  if constexpr (WAVES == 1) {
    a = group_sum(a, lanes);
    b = group_sum(b, lanes);
  } else {
    a = group_sum(a, kWave);
    b = group_sum(b, kWave);
    __syncthreads();
    if (lane_id() == 0) lds[2 * wave_in_block()] = a, lds[2 * wave_in_block() + 1] = b;
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) a += lds[2 * w], b += lds[2 * w + 1];
  }
}

// The same with one barrier: two parts of LDS take turns, and whoever writes one again has met the others behind their reads of it.
template <int WAVES>
struct RowSums {
  float* lds;  // [4 WAVES]
  int turn;
  __device__ __forceinline__ explicit RowSums(float* lds_) : lds(lds_), turn(0) {}
  __device__ __forceinline__ void operator()(float& a, float& b, int lanes) {
    a = group_sum(a, WAVES == 1 ? lanes : kWave);
    b = group_sum(b, WAVES == 1 ? lanes : kWave);
    if constexpr (WAVES > 1) {
      float* const to = lds + turn * 2 * WAVES;
      turn ^= 1;
      if (lane_id() == 0) to[2 * wave_in_block()] = a, to[2 * wave_in_block() + 1] = b;
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) a += to[2 * w], b += to[2 * w + 1];
    }
  }
  __device__ __forceinline__ float operator()(float a, int lanes) {
    a = group_sum(a, WAVES == 1 ? lanes : kWave);
    if constexpr (WAVES > 1) {
      float* const to = lds + turn * 2 * WAVES;
      turn ^= 1;
      if (lane_id() == 0) to[wave_in_block()] = a;
      __syncthreads();
      a = 0.f;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) a += to[w];
    }
    return a;
  }
};

template <int WAVES> constexpr int kNormBlock = WAVES == 1 ? kBlock : WAVES * kWave;

// which rows a block takes: its first group's row, rows from group to group of the grid, and this lane's group in the block
template <int WAVES>
struct Rows {
  int64_t first, step;
  int lane, group;
  template <typename Shape>
  __device__ __forceinline__ explicit Rows(const Shape& sh) {
    if constexpr (WAVES == 1) {
      const int per_block = kBlock >> sh.lanes_log2;
      group = threadIdx.x >> sh.lanes_log2;
      lane = threadIdx.x & (sh.lanes - 1);
      first = (int64_t)blockIdx.x * per_block + group;
      step = (int64_t)gridDim.x * per_block;
    } else {
      group = 0;
      lane = threadIdx.x;
      first = blockIdx.x;
      step = gridDim.x;
    }
  }
  template <typename Shape>
  __device__ __forceinline__ int lanes(const Shape& sh) const { return WAVES == 1 ? sh.lanes : WAVES * kWave; }
};

}  // namespace coop
