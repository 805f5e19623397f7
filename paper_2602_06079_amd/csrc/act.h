// The activations and their slopes, in fp32.
#pragma once
#include "device_util.h"

namespace canz {

constexpr bool act_known(int32_t act) { return act >= CANZ_ACT_NONE && act <= CANZ_ACT_RELU; }

struct ActValue {
  float value, slope;   // act(z), act'(z)
};

// e^x for the sigmoid: v_exp_f32 is good to one step, and the product in front of it is off by at most |x| 2^-24 2, that is 1.2e-6 of a result of
// e^-10 and less of a larger one.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }

// Phi(z) and e^(-z^2 / 2).  With x = |z| / sqrt 2 the tail Phi(-|z|) is e^(-x^2) f(x), f(x) = e^(x^2) erfc(x) / 2, which is smooth in t = 1 / (1 + 0.4 x): a polynomial of degree 9
// in t, fitted here by weighted least squares over x in 0 .. 11, is off by 3.6e-8 of it at most (2e-7 in fp32), so that Phi keeps its relative accuracy far below 0.  Behind x = 11 the
// exponential is 0.  The library's erfc takes all of its ranges where lanes differ: 4096 x 25600 x 5120 with GELU 1017 us with it, without an activation 846.
struct Normal {
  float phi, density;   // density: without 1 / sqrt(2 pi)
};
__device__ __forceinline__ Normal normal(float z) {
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(__builtin_fabsf(z), 0.28284271247461901f, 1.f));
  const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
  float f = 0.015846358612179756f;
  f = __builtin_fmaf(f, t, -0.045312441885471344f);
  f = __builtin_fmaf(f, t, -0.013677749782800674f);
  f = __builtin_fmaf(f, t, 0.11437621712684631f);
  f = __builtin_fmaf(f, t, -0.01534305326640606f);
  f = __builtin_fmaf(f, t, 0.12450025230646133f);
  f = __builtin_fmaf(f, t, 0.09197775274515152f);
  f = __builtin_fmaf(f, t, 0.11500431597232819f);
  f = __builtin_fmaf(f, t, 0.11261897534132004f);
  f = __builtin_fmaf(f, t, 9.37712593440665e-06f);
  f *= e;
  return Normal{z > 0.f ? 1.f - f : f, e};
}

template <int ACT>
__device__ __forceinline__ ActValue act_both(float z) {
  if constexpr (ACT == CANZ_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
    const float v = z * p;
    return ActValue{v, __builtin_fmaf(v, 1.f - p, p)};
  } else if constexpr (ACT == CANZ_ACT_GELU) {
    const Normal n = normal(z);
    return ActValue{z * n.phi, __builtin_fmaf(z * 0.39894228040143268f, n.density, n.phi)};
  } else if constexpr (ACT == CANZ_ACT_RELU) {
    const bool nan = z != z;
    return ActValue{nan ? z : __builtin_fmaxf(z, 0.f), nan ? z : z > 0.f ? 1.f : 0.f};
  } else {
    return ActValue{z, 1.f};
  }
}

}  // namespace canz
