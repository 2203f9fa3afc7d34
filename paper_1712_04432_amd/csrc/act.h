// Activations of a fully connected layer and their derivatives, in fp32.
#pragma once

#include "common.h"

namespace imbd {

// e^x to a few units in the last place, 0 where that is under the smallest normal number; 1 / x likewise.
__device__ __forceinline__ float quick_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }
__device__ __forceinline__ float quick_rcp(float x) { return __builtin_amdgcn_rcpf(x); }

// The standard normal distribution's tail beyond u >= 0, given e = exp(-u^2 / 2): e times a rational function of u, whose
// coefficients are a least-maximum fit of exp(u^2 / 2) * tail in t = 1 / (1 + u / 4) over all u (relative error 4.7e-8 with the
// coefficients as rounded, 4e-7 as evaluated in fp32; tests/test_act_fit.py). Nothing cancels, so the tail keeps its
// digits however small it is but for those that e loses to its argument's rounding: its relative error grows as 2^-24 u^2.
__device__ __forceinline__ float normal_tail(float u, float e) {
  const float t = quick_rcp(fmaf(0.25f, u, 1.f));
  float p = 0.0197819881f;
  p = fmaf(p, t, -0.0808772147f);
  p = fmaf(p, t, 0.0955969095f);
  p = fmaf(p, t, -0.0317173563f);
  p = fmaf(p, t, 0.0636990219f);
  p = fmaf(p, t, 0.0589751787f);
  p = fmaf(p, t, 0.0816031024f);
  p = fmaf(p, t, 0.0934663564f);
  p = fmaf(p, t, 0.0997364298f);
  p = fmaf(p, t, 0.0997355655f);
  return e * (p * t);
}
// 1 / (1 + e^-x), exact relatively on both sides
__device__ __forceinline__ float logistic(float x) { return quick_rcp(1.f + quick_exp(-x)); }

constexpr float GELU_C = 1.59576912160573071176f;  // 2 sqrt(2 / pi)
constexpr float GELU_A = 0.044715f;

// GELU: z times the normal distribution up to z. GELU_TANH: with 1/2 (1 + tanh(y)) = logistic(2 y) in its place,
// y = sqrt(2 / pi) (z + 0.044715 z^3). SILU: z logistic(z). A NaN stays one (in RELU's derivative it counts as not positive).
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
  if constexpr (ACT == IMBD_ACT_RELU) return z < 0.f ? 0.f : z;
  if constexpr (ACT == IMBD_ACT_GELU) {
    const float q = normal_tail(fabsf(z), quick_exp(-0.5f * z * z));
    return z * (z < 0.f ? q : 1.f - q);
  }
  if constexpr (ACT == IMBD_ACT_GELU_TANH) return z * logistic(GELU_C * fmaf(GELU_A * z * z, z, z));
  if constexpr (ACT == IMBD_ACT_SILU) return z * logistic(z);
  return z;
}
// v times the derivative at z.
template <int ACT>
__device__ __forceinline__ float act_slope(float v, float z) {
  if constexpr (ACT == IMBD_ACT_RELU) return z > 0.f ? v : 0.f;
  if constexpr (ACT == IMBD_ACT_GELU) {
    const float e = quick_exp(-0.5f * z * z), q = normal_tail(fabsf(z), e);
    const float zc = fminf(fmaxf(z, -64.f), 64.f);  // (past it e is 0)
    return v * fmaf(zc * 0.398942280401432677940f, e, z < 0.f ? q : 1.f - q);
  }
  if constexpr (ACT == IMBD_ACT_GELU_TANH) {
    const float p = logistic(GELU_C * fmaf(GELU_A * z * z, z, z));
    const float zc = fminf(fmaxf(z, -64.f), 64.f);  // (past it p (1 - p) is 0)
    return v * fmaf(zc * p * (1.f - p), GELU_C * fmaf(3.f * GELU_A * zc, zc, 1.f), p);
  }
  if constexpr (ACT == IMBD_ACT_SILU) {
    const float p = logistic(z);
    return v * fmaf(p * (1.f - p), fminf(fmaxf(z, -1024.f), 1024.f), p);
  }
  return v;
}

// f(the activation as a constant).
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  if (act == IMBD_ACT_RELU) f(std::integral_constant<int, IMBD_ACT_RELU>{});
  else if (act == IMBD_ACT_GELU) f(std::integral_constant<int, IMBD_ACT_GELU>{});
  else if (act == IMBD_ACT_GELU_TANH) f(std::integral_constant<int, IMBD_ACT_GELU_TANH>{});
  else if (act == IMBD_ACT_SILU) f(std::integral_constant<int, IMBD_ACT_SILU>{});
}
template <int N>
__device__ __forceinline__ void apply_act(int act, float (&v)[N]) {
  with_act(act, [&](auto tag) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_value<decltype(tag)::value>(v[i]);
  });
}
template <int N>
__device__ __forceinline__ void apply_slope(int act, float (&v)[N], const float (&z)[N]) {
  with_act(act, [&](auto tag) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = act_slope<decltype(tag)::value>(v[i], z[i]);
  });
}

}  // namespace imbd
