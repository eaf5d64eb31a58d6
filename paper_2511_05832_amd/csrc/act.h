// Activations of the linear layer and their derivatives, in fp32.
#pragma once

#include "hla_internal.h"

namespace hla {

// The normal distribution's tail Phi(-|z|) and density, from one exponential: erfc by
// Abramowitz & Stegun, Handbook of Mathematical Functions, 7.1.26 (|error| < 1.5e-7),
// erfc(x) = t (a1 + t (a2 + ...)) e^{-x^2}, t = 1 / (1 + p x), x = |z| / sqrt 2. About
// 14 operations beside erff's 40; taken for bf16 results, whose half step is 2^-8.
__device__ __forceinline__ float normal_tail(float z, float &density) {
  const float e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);   // e^{-z^2 / 2}
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
  float p = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  p = __builtin_fmaf(p, t, 1.421413741f);
  p = __builtin_fmaf(p, t, -0.284496736f);
  p = __builtin_fmaf(p, t, 0.254829592f);
  density = 0.39894228040143268f * e;
  return 0.5f * p * t * e;
}

// gelu(z) = max(z, 0) - |z| Phi(-|z|), with log2 Phi(-a) a polynomial: smooth, from -1 at 0
// to the parabola of the tail, so one exponential and no reciprocal. The coefficients are
// the minimax fit on 0 <= a <= 8 of the larger of the tail's error over 3e-7 and its
// relative error over 1e-4 (a linear programme on 2400 points); Phi is within 3.1e-7, and
// gelu within 1e-4 of itself down to 1e-8, against bf16's half step of 2^-8. From 8 to the
// 64 that |z| is taken to, the polynomial stays below -50 (it rises from -169 at 18 to -90 at
// 25), so Phi is nothing. 12 instructions, 7.1.26 takes 17 here, and a layer's epilogue is
// bound by their issue.
// |z| is taken up to 64: inf * 0 must not be formed. (minimum and maximum hand NaN on.)
__device__ __forceinline__ float gelu_fast(float z) {
  const float a = __builtin_elementwise_minimum(__builtin_fabsf(z), 64.f);
  float q = __builtin_fmaf(-7.49217696e-7f, a, 4.20198360e-5f);
  q = __builtin_fmaf(q, a, -7.97152815e-4f);
  q = __builtin_fmaf(q, a, 8.08079023e-3f);
  q = __builtin_fmaf(q, a, -5.33045511e-2f);
  q = __builtin_fmaf(q, a, -4.58911025e-1f);
  q = __builtin_fmaf(q, a, -1.15114427f);
  q = __builtin_fmaf(q, a, -0.999999204f);
  return __builtin_fmaf(-a, __builtin_amdgcn_exp2f(q), __builtin_elementwise_maximum(z, 0.f));
}

// EXACT: fp32 results.
template <bool EXACT>
__device__ __forceinline__ float normal_cdf(float z, float &density) {
  if constexpr (EXACT) {
    density = 0.39894228040143268f * expf(-0.5f * z * z);
    return 0.5f * erfcf(-0.70710678118654752f * z);
  } else {
    const float tail = normal_tail(z, density);
    return z < 0.f ? tail : 1.f - tail;
  }
}

// 1 / (1 + e^{-z}). For z below -88 the exponential is inf and the result 0.
template <bool EXACT>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (EXACT) return 1.f / (1.f + expf(-z));
  else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.4426950408889634f * z));
}

// gelu_tanh(z) = z / 2 (1 + tanh u) = z logistic(2 u), u = sqrt(2 / pi) (z + 0.044715 z^3).
constexpr float kGeluC = 0.79788456080286536f, kGeluA = 0.044715f;

// (beyond 30 the derivative is 0 or 1, and z^2 must not overflow)
template <bool EXACT>
__device__ __forceinline__ float gelu_tanh_grad(float z) {
  const float s = logistic<EXACT>(2.f * kGeluC * __builtin_fmaf(kGeluA * z * z, z, z));
  const float g = __builtin_fmaf(z * s * (1.f - s), 2.f * kGeluC * __builtin_fmaf(3.f * kGeluA * z, z, 1.f), s);
  return fabsf(z) > 30.f ? (z > 0.f ? 1.f : 0.f) : g;
}

// Past these a slope, or gelu below, has reached its limit (Phi(-64) and 1 / (1 + e^200) are 0
// in fp32), and z goes no further, so that inf * 0 is not formed. NaN is handed on. (The
// other activations are NaN at z = -inf: holding z there, too, costs a layer of 16384 x 4096
// results in bf16 146 -> 150 us with silu, one instruction a result.)
constexpr float kFarGelu = 64.f, kFarSilu = 200.f;
__device__ __forceinline__ float within(float z, float most) {
  return __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -most), most);
}

// z[e] = act(z[e]) for N values (one branch for all of them).
template <bool EXACT, int N>
__device__ __forceinline__ void apply_act(int act, float (&z)[N]) {
  float density;
  if (act == HLA_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = z[e] > 0.f ? z[e] : (z[e] != z[e] ? z[e] : 0.f);
  } else if (act == HLA_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (EXACT) z[e] = __builtin_elementwise_maximum(z[e], -kFarGelu) * normal_cdf<true>(z[e], density);
      else z[e] = gelu_fast(z[e]);
    }
  } else if (act == HLA_ACT_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      if constexpr (EXACT) {
        z[e] *= logistic<true>(2.f * kGeluC * __builtin_fmaf(kGeluA * z[e] * z[e], z[e], z[e]));
      } else {
        constexpr float k = -1.4426950408889634f * 2.f * kGeluC;
        const float u = z[e] * __builtin_fmaf(k * kGeluA, z[e] * z[e], k);
        z[e] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(u));
      }
    }
  } else if (act == HLA_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] *= logistic<EXACT>(z[e]);
  }
}

// z[e] = act'(z[e])
template <bool EXACT, int N>
__device__ __forceinline__ void apply_grad(int act, float (&z)[N]) {
  if (act == HLA_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = z[e] > 0.f ? 1.f : 0.f;
  } else if (act == HLA_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float density;
      z[e] = within(z[e], kFarGelu);
      const float cdf = normal_cdf<EXACT>(z[e], density);
      z[e] = __builtin_fmaf(z[e], density, cdf);
    }
  } else if (act == HLA_ACT_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = gelu_tanh_grad<EXACT>(z[e]);
  } else if (act == HLA_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      z[e] = within(z[e], kFarSilu);
      const float s = logistic<EXACT>(z[e]);
      z[e] = s * __builtin_fmaf(z[e], 1.f - s, 1.f);
    }
  }
}

}  // namespace hla
