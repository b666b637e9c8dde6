// Elements of the learning operators' tensors: fp32, fp16 and bf16 in memory, fp32 in registers.
#pragma once
#include "device_utils.h"

namespace coop {

template <int T> struct Element;
template <> struct Element<COOP_F32> { typedef float M; };
template <> struct Element<COOP_F16> { typedef _Float16 M; };
template <> struct Element<COOP_BF16> { typedef __bf16 M; };

inline int element_bytes(int dtype) { return dtype == COOP_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == COOP_F32 || dtype == COOP_F16 || dtype == COOP_BF16; }
inline bool aligned_for(const void* p, int dtype) { return ((uintptr_t)p & (uintptr_t)(element_bytes(dtype) - 1)) == 0; }

// E neighbouring elements of type T (E a power of two, at most 16 bytes), at any alignment that the type itself allows
template <int T, int E>
struct Pack {
  typedef typename Element<T>::M M;
  static constexpr int kBytes = E * (int)sizeof(M);
  typedef typename RowVec<kBytes>::T Raw;
  M x[E];
  static __device__ __forceinline__ Pack load(const void* p) {
    return __builtin_bit_cast(Pack, *reinterpret_cast<const typename RowVec<kBytes>::U*>(p));
  }
  static __device__ __forceinline__ Pack load_nt(const void* p) { return __builtin_bit_cast(Pack, row_load_nt<kBytes>((const char*)p)); }
  __device__ __forceinline__ void store(void* p) const { *reinterpret_cast<typename RowVec<kBytes>::U*>(p) = __builtin_bit_cast(Raw, *this); }
  __device__ __forceinline__ void store_nt(void* p) const { row_store_nt<kBytes>((char*)p, __builtin_bit_cast(Raw, *this)); }
  __device__ __forceinline__ void get(float (&f)[E]) const {
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = (float)x[i];
  }
  // rounded to nearest, ties to even
  __device__ __forceinline__ void set(const float (&f)[E]) {
#pragma unroll
    for (int i = 0; i < E; ++i) x[i] = (M)f[i];
  }
};

// E neighbouring elements as fp32, and back, 16 bytes at a time where they are longer than that
template <int T, int E>
__device__ __forceinline__ void load_elements(const void* p, float (&f)[E]) {
  constexpr int N = E * (int)sizeof(typename Element<T>::M) <= 16 ? E : 16 / (int)sizeof(typename Element<T>::M);
#pragma unroll
  for (int i = 0; i < E; i += N) {
    const Pack<T, N> x = Pack<T, N>::load((const char*)p + i * (int)sizeof(typename Element<T>::M));
#pragma unroll
    for (int e = 0; e < N; ++e) f[i + e] = (float)x.x[e];
  }
}
template <int T, int E>
__device__ __forceinline__ void store_elements(void* p, const float (&f)[E]) {
  constexpr int N = E * (int)sizeof(typename Element<T>::M) <= 16 ? E : 16 / (int)sizeof(typename Element<T>::M);
#pragma unroll
  for (int i = 0; i < E; i += N) {
    Pack<T, N> x;
#pragma unroll
    for (int e = 0; e < N; ++e) x.x[e] = (typename Element<T>::M)f[i + e];
    x.store((char*)p + i * (int)sizeof(typename Element<T>::M));
  }
}

// Sum over each aligned group of `lanes` lanes (a power of two up to 64); every lane of the group has it.
__device__ __forceinline__ float group_sum(float v, int lanes) {
#pragma unroll
  for (int off = 1; off < kWave; off <<= 1)
    if (off < lanes) v += __shfl_xor(v, off, kWave);
  return v;
}

// Calls f with the dtype as a compile-time constant; false for one that is not known.
template <typename F>
inline bool with_dtype(int dtype, F&& f) {
  switch (dtype) {
    case COOP_F32: f(std::integral_constant<int, COOP_F32>()); return true;
    case COOP_F16: f(std::integral_constant<int, COOP_F16>()); return true;
    case COOP_BF16: f(std::integral_constant<int, COOP_BF16>()); return true;
  }
  return false;
}

}  // namespace coop
