// The activations and their slopes, in fp32.
#pragma once
#include "device_util.h"

namespace canz {

constexpr bool act_known(int32_t act) { return act >= CANZ_ACT_NONE && act <= CANZ_ACT_RELU; }

struct ActValue {
  float value, slope;   // act(z), act'(z)
};

// e^x for the sigmoid and the normal density: v_exp_f32 is good to one step, and the product in front of it is off by at most |x| 2^-24 2, that is 1.2e-6 of a result of
// e^-10 and less of a larger one.
__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896f); }

// GELU.  Phi(z) = erfc(-z / sqrt 2) / 2, which keeps its relative accuracy where z is far below 0.
template <int ACT>
__device__ __forceinline__ ActValue act_both(float z) {
  if constexpr (ACT == CANZ_ACT_SILU) {
    const float p = __builtin_amdgcn_rcpf(1.f + exp_fast(-z));
    const float v = z * p;
    return ActValue{v, __builtin_fmaf(v, 1.f - p, p)};
  } else if constexpr (ACT == CANZ_ACT_GELU) {
    const float p = 0.5f * erfcf(z * -0.70710678118654752f);
    return ActValue{z * p, __builtin_fmaf(z * 0.39894228040143268f, exp_fast(-0.5f * z * z), p)};
  } else if constexpr (ACT == CANZ_ACT_RELU) {
    const bool nan = z != z;
    return ActValue{nan ? z : __builtin_fmaxf(z, 0.f), nan ? z : z > 0.f ? 1.f : 0.f};
  } else {
    return ActValue{z, 1.f};
  }
}

}  // namespace canz
