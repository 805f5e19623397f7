// Rounding of a block of 32 elements, shared by the kernels that make images and those that round an operand on its way.
//
// With E the biased exponent of the largest magnitude, the floor rule takes the scale byte E - 2, the ceil rule one more where the
// mantissa is above 1.5, both at least 0 (2^-127); the ceil rule's stops at 252 (2^125), where the floor rule's ends by itself.  Division by X
// is exact, and the conversion instructions round to the nearest value, ties to the even code, at most 6 (v_cvt_scalef32_pk_fp4_*: they read the
// exponent field of their scale alone, so that byte << 23 is 2^(byte - 127) for every byte).
#pragma once
#include "device_util.h"

namespace canz {

constexpr unsigned MX_NONFINITE = 0x7F800000u;   // magnitudes with these bits or above are infinite or NaN
constexpr unsigned MX_SCALE_NAN = 255u;
constexpr int MX_MAX_SCALE = 252;                // six times 2^125 is the largest value that fp32 holds

typedef __bf16 mx_bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned mx_magnitude(float v) { return __builtin_bit_cast(unsigned, v) & 0x7FFFFFFFu; }
// scale byte of a block whose largest magnitude has the bits `amax`
__device__ __forceinline__ unsigned mx_scale_byte(unsigned amax, int ceil) {
  // without branches: the lanes of a wavefront have blocks of their own
  const int up = ceil & static_cast<int>((amax & 0x7FFFFFu) > 0x400000u);
  const int e = min(max(static_cast<int>(amax >> 23) - 2 + up, 0), MX_MAX_SCALE);
  return amax >= MX_NONFINITE ? MX_SCALE_NAN : static_cast<unsigned>(e);
}
__device__ __forceinline__ float mx_scale_value(unsigned byte) { return __builtin_bit_cast(float, byte << 23); }

}  // namespace canz
