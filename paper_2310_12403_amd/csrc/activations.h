// Activations of the dense operators and their slopes, in 32 bits.
#pragma once
#include <type_traits>

#include "device_utils.h"

namespace coop {

// Phi(z), the normal distribution's, and e = exp(-z^2 / 2).  With x = |z| / sqrt 2, exp(x^2) erfc(x) = t P(t) for t = 1 / (1 + 0.355 x): P of
// degree 9, fitted for the least relative error (4e-8 for x up to 200), so that the tail is as exact as the middle but for the
// exponential's argument (2^-24 z^2 / 2).  Some 20 instructions; 1 + erf would lose the tail to cancellation, and erfc costs three times that.
__device__ __forceinline__ float normal_cdf(float z, float* e_out) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(fabsf(z), 0.355f * 0.70710678118654752f, 1.f));
  float p = 0.0404977f;
  p = __builtin_fmaf(p, t, -0.1631299f);
  p = __builtin_fmaf(p, t, 0.19071296f);
  p = __builtin_fmaf(p, t, -0.06556422f);
  p = __builtin_fmaf(p, t, 0.12849507f);
  p = __builtin_fmaf(p, t, 0.11705923f);
  p = __builtin_fmaf(p, t, 0.16378647f);
  p = __builtin_fmaf(p, t, 0.18756457f);
  p = __builtin_fmaf(p, t, 0.20029088f);
  p = __builtin_fmaf(p, t, 0.20028726f);
  const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  const float q = 0.5f * (p * t) * e;
  *e_out = e;
  return z < 0.f ? q : 1.f - q;
}

__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504088896341f)); }

__device__ __forceinline__ float act_value(float z, int act) {
  if (act == COOP_ACT_RELU) return z > 0.f ? z : z == z ? 0.f : z;  // (a NaN stays one)
  if (act == COOP_ACT_GELU) {
    float e;
    return z * normal_cdf(z, &e);
  }
  if (act == COOP_ACT_SILU) return z * logistic(z);
  return z;
}

// *value: act(z); the result: its slope.  (relu's at 0 is 0.)
__device__ __forceinline__ float act_slope(float z, int act, float* value) {
  if (act == COOP_ACT_RELU) {
    *value = z > 0.f ? z : z == z ? 0.f : z;
    return z > 0.f ? 1.f : z == z ? 0.f : z;
  }
  if (act == COOP_ACT_GELU) {
    float e;
    const float p = normal_cdf(z, &e);
    *value = z * p;
    return __builtin_fmaf(z * 0.39894228040143268f, e, p);
  }
  if (act == COOP_ACT_SILU) {
    const float p = logistic(z);
    *value = z * p;
    return p * __builtin_fmaf(z, 1.f - p, 1.f);
  }
  *value = z;
  return 1.f;
}

// The same of E values, in their places; which activation it is, is asked once.
template <int E>
__device__ __forceinline__ void act_values(float (&z)[E], int act) {
  const auto all = [&](auto a) {
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = act_value(z[e], decltype(a)::value);
  };
  if (act == COOP_ACT_GELU) all(std::integral_constant<int, COOP_ACT_GELU>());
  else if (act == COOP_ACT_SILU) all(std::integral_constant<int, COOP_ACT_SILU>());
  else if (act == COOP_ACT_RELU) all(std::integral_constant<int, COOP_ACT_RELU>());
}
// z: the slopes in its place; value: act(z)
template <int E>
__device__ __forceinline__ void act_slopes(float (&z)[E], float (&value)[E], int act) {
  const auto all = [&](auto a) {
#pragma unroll
    for (int e = 0; e < E; ++e) z[e] = act_slope(z[e], decltype(a)::value, &value[e]);
  };
  if (act == COOP_ACT_GELU) all(std::integral_constant<int, COOP_ACT_GELU>());
  else if (act == COOP_ACT_SILU) all(std::integral_constant<int, COOP_ACT_SILU>());
  else if (act == COOP_ACT_RELU) all(std::integral_constant<int, COOP_ACT_RELU>());
  else all(std::integral_constant<int, COOP_ACT_NONE>());
}

}  // namespace coop
