// An operand in fp32 as 16-bit planes.
#pragma once
#include "mfma_device.h"

namespace lq {

// 2^s that brings a magnitude with these bits below 2^14, as an exponent: fp16 then holds hi to 11 bits and lo to 11 more for
// everything within 2^-17 of the largest, and what is smaller to 2^-39 of it.  1 for a magnitude of zero.
__device__ __forceinline__ int half_exponent(uint32_t bits) {
  const int e = (int)(bits >> 23) - 127;                 // magnitude < 2^(e + 1)
  return bits == 0 ? 0 : e < -112 ? 125 : 13 - e;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 .. 127
__device__ __forceinline__ uint32_t finite_magnitude(float v) {
  const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}

// The exponent for an operand whose largest magnitude is the largest of `count` words.
__device__ __forceinline__ int half_exponent_of(const uint32_t* __restrict__ tops, int count) {
  uint32_t top = 0;
  for (int i = 0; i < count; ++i) top = max(top, tops[i]);
  return half_exponent(top);
}

struct HalfPair { _Float16 hi, lo; };
__device__ __forceinline__ HalfPair split_half(float v) {
  const _Float16 h = (_Float16)v;
  return {h, (_Float16)(v - (float)h)};
}
// v = p[0] + p[1] + p[2] + O(2^-25 v).
__device__ __forceinline__ void split_bf16_3(floatx2 v, bf16x2 (&p)[3]) {
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    p[k] = __builtin_convertvector(v, bf16x2);
    v = v - __builtin_convertvector(p[k], floatx2);
  }
}

}  // namespace lq
