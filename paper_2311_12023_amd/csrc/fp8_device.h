// e4m3 codes and their scales.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "mfma_device.h"

namespace lq {

typedef int intx8 __attribute__((ext_vector_type(8)));

// Accumulators of products hold 2^30 times the result, so that the product of two small scales stays a normal number.
constexpr float FP8_LIFT = 0x1p30f, FP8_DROP = 0x1p-30f;
// The lifted product of two scales (NaN where one is): the lift goes to `s` unless that is large, so that it is inf only where the product
// of both is 2^98 or more.
__device__ __forceinline__ float fp8_lifted(float s, float f) {
  const int lift = fabsf(s) >= 0x1p60f ? 0 : 30;
  return __builtin_amdgcn_ldexpf(s, lift) * __builtin_amdgcn_ldexpf(f, 30 - lift);
}

// Magnitudes are compared as bit patterns: NaN ranks above inf, inf above all numbers.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale of a block whose largest magnitude has the bits `top`: the largest code is 448.  The quotient, rounded: with y = fl(1 / 448) and
// q = fl(a y), the rest a - 448 q is a float, and fl(q + rest y) is fl(a / 448) (Markstein, 1990) where it is normal; what is not
// becomes 2^-126.  Three instructions for the ten of a division.
__device__ __forceinline__ float fp8_scale(uint32_t top) {
  const float a = __uint_as_float(top), y = 1.0f / 448.0f, q = a * y;
  const float s = fmaxf(fmaf(fmaf(-448.0f, q, a), y, q), 0x1p-126f);
  return top >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : s;
}
// fl(1 / s) of a scale (2^-126 .. 2^120, or NaN): the hardware's reciprocal, which is within a unit in the last place, and one Newton step.
// From an estimate a whole unit off the step ends next to the rounded quotient for 31 scales' fractions; this chip's estimates do not lead
// there: the tests quantize blocks of all 2^23 fractions of amax.  Powers of two change nothing in this range.
__device__ __forceinline__ float fp8_inverse(float s) {
  const float y = __builtin_amdgcn_rcpf(s);
  return fmaf(fmaf(-s, y, 1.0f), y, y);
}

// Codes of two neighbours in the lower or upper half of `old`.  |a|, |b| <= 448 (1 + 2^-22), which rounds to 448: nothing saturates.
template <bool HIGH>
__device__ __forceinline__ uint32_t fp8_pair(float a, float b, uint32_t old) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, (int)old, HIGH);
}
__device__ __forceinline__ uint32_t fp8_four(float a, float b, float c, float d) { return fp8_pair<true>(c, d, fp8_pair<false>(a, b, 0)); }

// Values of the four codes of a word.
__device__ __forceinline__ floatx4 fp8_values(uint32_t w) {
  const floatx2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return floatx4{lo[0], lo[1], hi[0], hi[1]};
}

}  // namespace lq
