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

template <bool EXACT>
__device__ __forceinline__ float act_of(int act, float z) {
  switch (act) {
    case HLA_ACT_RELU: return z > 0.f ? z : (z != z ? z : 0.f);
    case HLA_ACT_GELU: {
      float density;
      return z * normal_cdf<EXACT>(z, density);
    }
    case HLA_ACT_GELU_TANH: return z * logistic<EXACT>(2.f * kGeluC * __builtin_fmaf(kGeluA * z * z, z, z));
    case HLA_ACT_SILU: return z * logistic<EXACT>(z);
    default: return z;
  }
}

template <bool EXACT>
__device__ __forceinline__ float act_grad(int act, float z) {
  switch (act) {
    case HLA_ACT_RELU: return z > 0.f ? 1.f : 0.f;
    case HLA_ACT_GELU: {
      float density;
      const float cdf = normal_cdf<EXACT>(z, density);
      return __builtin_fmaf(z, density, cdf);
    }
    case HLA_ACT_GELU_TANH: {
      // (beyond 30 the derivative is 0 or 1, and z^2 must not overflow)
      if (fabsf(z) > 30.f) return z > 0.f ? 1.f : 0.f;
      const float s = logistic<EXACT>(2.f * kGeluC * __builtin_fmaf(kGeluA * z * z, z, z));
      return __builtin_fmaf(z * s * (1.f - s), 2.f * kGeluC * __builtin_fmaf(3.f * kGeluA * z, z, 1.f), s);
    }
    case HLA_ACT_SILU: {
      const float s = logistic<EXACT>(z);
      return s * __builtin_fmaf(z, 1.f - s, 1.f);
    }
    default: return 1.f;
  }
}

}  // namespace hla
