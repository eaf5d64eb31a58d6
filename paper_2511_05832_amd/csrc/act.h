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

// gelu(z) = max(z, 0) - |z| Phi(-|z|) with the same formula. |z| is taken up to 88, where
// the tail is 0 already: inf * 0 must not be formed. (v_med3 takes one instruction where
// fminf takes two; a NaN comes back through the exponential.)
__device__ __forceinline__ float gelu_fast(float z) {
  const float a = __builtin_amdgcn_fmed3f(fabsf(z), 0.f, 88.f);
  float density;
  const float tail = normal_tail(z, density);
  return __builtin_fmaf(-a, tail, __builtin_amdgcn_fmed3f(z, 0.f, __builtin_inff()));
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
      if constexpr (EXACT) z[e] *= normal_cdf<true>(z[e], density);
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
      const float cdf = normal_cdf<EXACT>(z[e], density);
      z[e] = __builtin_fmaf(z[e], density, cdf);
    }
  } else if (act == HLA_ACT_GELU_TANH) {
#pragma unroll
    for (int e = 0; e < N; ++e) z[e] = gelu_tanh_grad<EXACT>(z[e]);
  } else if (act == HLA_ACT_SILU) {
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float s = logistic<EXACT>(z[e]);
      z[e] = s * __builtin_fmaf(z[e], 1.f - s, 1.f);
    }
  }
}

}  // namespace hla
