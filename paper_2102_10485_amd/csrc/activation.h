// The activations of the products' epilogues, and their derivatives.
//
//   GAN_ACT_RELU  max(z, 0)         1 above zero, 0 at zero and below
//   GAN_ACT_GELU  z Phi(z)          Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi)       (Phi: the normal distribution's; no approximation by tanh)
//   GAN_ACT_SILU  z s(z)            s(z) (1 + z (1 - s(z))),  s(z) = 1 / (1 + exp(-z))
//
// At infinity they are their limits; NaN stays NaN.
#pragma once

#include "operators.h"

namespace gan {

__device__ __forceinline__ float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }             // (to one ulp)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Phi(z), and exp(-z^2 / 2).  NEAR: for results that are rounded to bf16 (half a step is 2^-9 of the value): the tail is exp(-z^2 / 2) times a polynomial of 1 / (1 + 0.305 |z|),
// fitted to exp(z^2 / 2) erfc(z / sqrt 2) / 2 on [0, 13] with the least largest relative error, 4.7e-6 (a seventh of the instructions of erfc).
template <bool NEAR>
__device__ __forceinline__ void normal_cdf(float z, float& phi, float& bell) {
  if constexpr (NEAR) {
    const float a = fabsf(z), t = reciprocal(fmaf(0.305f, a, 1.f));
    bell = exp2_fast(a * a * -0.72134752044448170f);              // 1 / (2 ln 2)
    float p = -0.0766185000538826f;
    p = fmaf(p, t, 0.20079532265663147f);
    p = fmaf(p, t, -0.0029916984494775534f);
    p = fmaf(p, t, 0.14002127945423126f);
    p = fmaf(p, t, 0.11680129170417786f);
    p = fmaf(p, t, 0.12199409306049347f);
    const float tail = p * t * bell;
    phi = z < 0.f ? tail : 1.f - tail;
  } else {
    phi = 0.5f * erfcf(z * -0.70710678118654752f);
    bell = expf(z * z * -0.5f);
  }
}
template <bool NEAR>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (NEAR) return reciprocal(1.f + exp2_fast(z * -1.44269504088896341f));
  else return 1.f / (1.f + expf(-z));
}

// the limits at -infinity are zeros: there the factor that vanishes is met by a finite one
template <bool NEAR>
__device__ __forceinline__ float gelu(float z) {
  float phi, bell;
  normal_cdf<NEAR>(z, phi, bell);
  return (z < -20.f ? -20.f : z) * phi;
}
template <bool NEAR>
__device__ __forceinline__ float gelu_slope(float z) {
  float phi, bell;
  normal_cdf<NEAR>(z, phi, bell);
  const float c = z < -20.f ? -20.f : z > 20.f ? 20.f : z;
  return fmaf(c * 0.39894228040143268f, bell, phi);               // 1 / sqrt(2 pi)
}
template <bool NEAR>
__device__ __forceinline__ float silu(float z) { return (z < -200.f ? -200.f : z) * logistic<NEAR>(z); }
template <bool NEAR>
__device__ __forceinline__ float silu_slope(float z) {
  const float s = logistic<NEAR>(z), c = z < -200.f ? -200.f : z > 200.f ? 200.f : z;
  return s * fmaf(c, 1.f - s, 1.f);
}

template <bool NEAR, int N>
__device__ __forceinline__ void activate(int act, float (&z)[N]) {
  if (act == GAN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];
  } else if (act == GAN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = gelu<NEAR>(z[i]);
  } else if (act == GAN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = silu<NEAR>(z[i]);
  }
}
// d *= the activation's derivative at z
template <bool NEAR, int N>
__device__ __forceinline__ void times_slope(int act, float (&d)[N], const float (&z)[N]) {
  if (act == GAN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = z[i] > 0.f ? d[i] : z[i] != z[i] ? z[i] : 0.f;
  } else if (act == GAN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= gelu_slope<NEAR>(z[i]);
  } else if (act == GAN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= silu_slope<NEAR>(z[i]);
  }
}

inline bool act_known(int act) { return act >= GAN_ACT_NONE && act <= GAN_ACT_SILU; }

}  // namespace gan
