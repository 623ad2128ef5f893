// The activations of the products' epilogues, and their derivatives.
//
//   GAN_ACT_RELU  max(z, 0)         1 above zero, 0 at zero and below
//   GAN_ACT_GELU  z Phi(z)          Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi)       (Phi: the normal distribution's; no approximation by tanh)
//   GAN_ACT_SILU  z s(z)            s(z) (1 + z (1 - s(z))),  s(z) = 1 / (1 + exp(-z))
//
// At infinity they are their limits; NaN stays NaN.  Results below 2^-119 may be zero: from z = -88.7 down, where SiLU is -2.6e-37, its exp(-z) is infinite in fp32, and the hardware's reciprocal, which
// results in bf16 take, has no numbers below 2^-126.
#pragma once

#include "operators.h"

namespace gan {

__device__ __forceinline__ float reciprocal(float x) { return __builtin_amdgcn_rcpf(x); }             // (to one ulp)
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// The normal distribution's tail beyond a = |z|, Phi(-a), and bell = exp(-a^2 / 2): bell times a polynomial of t = 1 / (1 + 0.305 a), fitted to exp(a^2 / 2) erfc(a / sqrt 2) / 2 on
// [0, 13] with the least largest relative error.
//   NEAR   six terms, 4.5e-6 (4.7e-6 in fp32): for results that are rounded to bf16 (half a step is 2^-8 of the value); 15 instructions, where erfc and exp take 80
//   else   eight terms, 1.27e-7 with the coefficients in fp32, which is two roundings of 2^-24: what an fp32 evaluation of any formula keeps where Phi is of size one.  Those of
//          the reciprocal, the exponential and the products come on top
//   EXACT  and the exponent a^2 / (2 ln 2) with the rounding errors of its products, which would cost a^2 roundings of the value
enum Accuracy { NEAR, FULL, EXACT };
template <Accuracy A>
__device__ __forceinline__ float normal_tail(float a, float& bell) {
  const float t = reciprocal(fmaf(0.305f, a, 1.f)), square = a * a, c = -0.72134752044448170f;         // 1 / (2 ln 2)
  const float arg = square * c;
  bell = exp2_fast(arg);
  if constexpr (A == EXACT) {
    float rest = fmaf(square, c, -arg) + fmaf(a, a, -square) * c + square * -9.6298149e-9f;           // (the last: what c leaves out)
    rest = square < 400.f ? rest : 0.f;
    bell = fmaf(bell, rest * 0.69314718055994531f, bell);
  }
  float p;
  if constexpr (A == NEAR) {
    p = -0.0766185000538826f;
    p = fmaf(p, t, 0.20079532265663147f);
    p = fmaf(p, t, -0.0029916984494775534f);
    p = fmaf(p, t, 0.14002127945423126f);
    p = fmaf(p, t, 0.11680129170417786f);
    p = fmaf(p, t, 0.12199409306049347f);
  } else {
    p = 0.03669889271259308f;
    p = fmaf(p, t, -0.15298710763454437f);
    p = fmaf(p, t, 0.18571491539478302f);
    p = fmaf(p, t, -0.037975069135427475f);
    p = fmaf(p, t, 0.12102078646421432f);
    p = fmaf(p, t, 0.10342112928628922f);
    p = fmaf(p, t, 0.12246678024530411f);
    p = fmaf(p, t, 0.12163973599672318f);
  }
  return p * t * bell;
}
template <Accuracy A>
__device__ __forceinline__ float logistic(float z) {
  if constexpr (A == EXACT) return 1.f / (1.f + expf(-z));
  else return reciprocal(1.f + exp2_fast(z * -1.44269504088896341f));
}

// z Phi(z) = max(z, 0) - |z| Phi(-|z|).  At infinity the factor that vanishes is met by a finite one.
template <Accuracy A>
__device__ __forceinline__ float gelu(float z) {
  float bell;
  const float tail = normal_tail<A>(fabsf(z), bell);
  return fmaf(-fminf(fabsf(z), 20.f), tail, fmaxf(z, 0.f));
}
template <Accuracy A>
__device__ __forceinline__ float gelu_slope(float z) {
  float bell;
  const float tail = normal_tail<A>(fabsf(z), bell), phi = z < 0.f ? tail : 1.f - tail;
  return fmaf(fminf(fmaxf(z, -20.f), 20.f) * 0.39894228040143268f, bell, phi);                        // 1 / sqrt(2 pi)
}
template <Accuracy A>
__device__ __forceinline__ float silu(float z) { return fmaxf(z, -200.f) * logistic<A>(z); }
template <Accuracy A>
__device__ __forceinline__ float silu_slope(float z) {
  const float s = logistic<A>(z);
  return s * fmaf(fminf(fmaxf(z, -200.f), 200.f), 1.f - s, 1.f);
}

template <Accuracy A, int N>
__device__ __forceinline__ void activate(int act, float (&z)[N]) {
  if (act == GAN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];
  } else if (act == GAN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = gelu<A>(z[i]);
  } else if (act == GAN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = silu<A>(z[i]);
  }
}
// d *= the activation's derivative at z
template <Accuracy A, int N>
__device__ __forceinline__ void times_slope(int act, float (&d)[N], const float (&z)[N]) {
  if (act == GAN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = z[i] > 0.f ? d[i] : z[i] != z[i] ? z[i] : 0.f;
  } else if (act == GAN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= gelu_slope<A>(z[i]);
  } else if (act == GAN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] *= silu_slope<A>(z[i]);
  }
}

inline bool act_known(int act) { return act >= GAN_ACT_NONE && act <= GAN_ACT_SILU; }

}  // namespace gan
