// The activations and their slopes, in fp32.
#pragma once
#include "device_util.h"

namespace canz {

constexpr bool act_known(int32_t act) { return act >= CANZ_ACT_NONE && act <= CANZ_ACT_RELU; }

struct ActValue {
  float value, slope;   // act(z), act'(z)
};

// FINE: for fp32 results of arguments that are given.  Without it the same forms lack a correction each: for results in bf16, whose rounding is off by up to 2^-8 = 3.9e-3, and for a product's z, which is off by more
// itself (1.9e-7 of its norm in 777 x 1531 x 1000).  In fp32 act(gate) up of 8192 x 8192 takes 390 us forward and back either way; in bf16 8192 x 12288 with GELU took 323 us without
// and 332 with its correction (and one more term), and the product of 4096 x 25600 x 5120 967 and 984.

// 1 / (1 + e^-z); with FINE SiLU is off by 2.8e-7 of itself at most.  x log2 e is rounded for the exponential, which counts |x| 2^-24 (without the correction SiLU is off by 9.7e-7 at -12 and 3.8e-6 at -85); what the
// rounding (of it and of log2 e) leaves out is exact in r and goes on as a factor of the power.  The factor's bounds matter where there is no r: an infinite argument, for which the power is 0 or infinite.
template <bool FINE>
__device__ __forceinline__ float sigmoid(float z) {
  constexpr float LOG2E = 1.4426950216293335f, LN2 = 0.69314718055994531f, REST = 1.3349758e-8f;   // REST: (log2 e - LOG2E) ln 2
  const float n = z * -LOG2E, power = __builtin_amdgcn_exp2f(n);
  if constexpr (!FINE) return __builtin_amdgcn_rcpf(1.f + power);
  const float r = __builtin_fmaf(z, -LOG2E, -n);
  const float w = __builtin_amdgcn_fmed3f(__builtin_fmaf(r, LN2, __builtin_fmaf(z, -REST, 1.f)), 0.999f, 1.001f);
  return __builtin_amdgcn_rcpf(__builtin_fmaf(power, w, 1.f));
}

// Phi(z) and e^(-z^2 / 2).  The tail Phi(-|z|) is e^(-z^2 / 2) f(z), f(z) = e^(z^2 / 2) erfc(|z| / sqrt 2) / 2, which is smooth in t = 1 / (1 + A |z|): a polynomial of degree 9
// in t, fitted here by weighted least squares over |z| in 0 .. 15.6, is off by 2.1e-8 of it at most with these coefficients (A = 11/32; 2.4e-8 with 1/4, 7e-8 with 3/8).  f changes by up to 2.3 times what t
// changes by, so that in fp32 its value is off by 5.4e-7 at most; FINE sets t right by what 1 - t (1 + A |z|) leaves, and then it is 2.6e-7 (z Phi(z) from -1/2 to 0: 2.9e-7, 7e-8 in the mean).  The exponential's argument is rounded twice, which counts
// up to z^2 2^-24 of Phi(-|z|): its relative accuracy falls from there on, as that of any form that squares z does.  Behind 15.6 the exponential is 0.
// The library's erfc takes all of its ranges where lanes differ: 4096 x 25600 x 5120 with GELU 1017 us with it, without an activation 846.
struct Normal {
  float phi, density;   // density: without 1 / sqrt(2 pi)
};
template <bool FINE>
__device__ __forceinline__ Normal normal(float z) {
  constexpr float A = 0.34375f;
  const float x = FINE ? __builtin_fminf(__builtin_fabsf(z), 16.f) : __builtin_fabsf(z);   // FINE: an infinite one would leave NaN
  float t = __builtin_amdgcn_rcpf(__builtin_fmaf(x, A, 1.f));
  if constexpr (FINE) t = __builtin_fmaf(t, __builtin_fmaf(-t, A * x, 1.f - t), t);
  const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  float f = -0.028713546693325043f;
  f = __builtin_fmaf(f, t, 0.14833438396453857f);
  f = __builtin_fmaf(f, t, -0.2812874913215637f);
  f = __builtin_fmaf(f, t, 0.20243380963802338f);
  f = __builtin_fmaf(f, t, -0.04788303002715111f);
  f = __builtin_fmaf(f, t, 0.11675199866294861f);
  f = __builtin_fmaf(f, t, 0.11549052596092224f);
  f = __builtin_fmaf(f, t, 0.1377772092819214f);
  f = __builtin_fmaf(f, t, 0.13709503412246704f);
  f = __builtin_fmaf(f, t, 1.0978608315781457e-06f);
  f *= e;
  return Normal{z > 0.f ? 1.f - f : f, e};
}

template <int ACT, bool FINE>
__device__ __forceinline__ ActValue act_both(float z) {
  if constexpr (ACT == CANZ_ACT_SILU) {
    const float p = sigmoid<FINE>(z);
    const float v = z * p;
    return ActValue{v, __builtin_fmaf(v, 1.f - p, p)};
  } else if constexpr (ACT == CANZ_ACT_GELU) {
    const Normal n = normal<FINE>(z);
    return ActValue{z * n.phi, __builtin_fmaf(z * 0.39894228040143268f, n.density, n.phi)};
  } else if constexpr (ACT == CANZ_ACT_RELU) {
    const bool nan = z != z;
    return ActValue{nan ? z : __builtin_fmaxf(z, 0.f), nan ? z : z > 0.f ? 1.f : 0.f};
  } else {
    return ActValue{z, 1.f};
  }
}

}  // namespace canz
