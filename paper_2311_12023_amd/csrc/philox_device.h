// The dropout mask: a counter-based generator, so that every kernel that meets an element works out for itself whether it is
// kept, and no mask is stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace lq {

// What decides which elements are kept and what they are multiplied by.
struct DropoutMask {
  uint64_t seed, offset;
  uint32_t cut;        // kept iff the element's 16 random bits are at least this: round(65536 p)
  float scale;         // 65536 / (65536 - cut); 0 where nothing is kept
};

// Philox4x32 with seven rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011; seven is the
// smallest count they report to pass every test of BigCrush, and a mask asks for no more than that).  Four words serve the eight
// elements of one group with 16 bits each: p is met to 2^-17, the factor is that of the rounded p, so the expectation stays
// exact.  14 products of 32 x 32 bits per eight elements; with 32 bits an element it would be 28.
struct PhiloxWords { uint32_t w[4]; };
__device__ __forceinline__ PhiloxWords philox_words(const DropoutMask& d, uint64_t group) {
  uint32_t c0 = (uint32_t)group, c1 = (uint32_t)(group >> 32), c2 = (uint32_t)d.offset, c3 = (uint32_t)(d.offset >> 32);
  uint32_t k0 = (uint32_t)d.seed, k1 = (uint32_t)(d.seed >> 32);
#pragma unroll
  for (int round = 0; round < 7; ++round) {
    const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
    const uint32_t n0 = (uint32_t)(b >> 32) ^ c1 ^ k0, n2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
    c1 = (uint32_t)b; c3 = (uint32_t)a; c0 = n0; c2 = n2;
    k0 += 0x9E3779B9u; k1 += 0xBB67AE85u;
  }
  return {{c0, c1, c2, c3}};
}
// Whether element j (0..7, a constant after unrolling) of the group is kept.
__device__ __forceinline__ bool philox_kept(const PhiloxWords& p, int j, uint32_t cut) {
  const uint32_t w = p.w[j >> 1];
  return ((j & 1) ? w >> 16 : w & 0xffffu) >= cut;
}

}  // namespace lq
