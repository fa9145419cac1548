// The order that the sampling kernel searches in: floats as whole numbers without gaps, and where its search looks next.
// Plain C++, so that the search can be followed on a CPU.
#pragma once

#include <cstdint>

#ifdef __CUDACC__
#define MQ_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define MQ_HOST_DEVICE inline
#endif

namespace mq {

// The bits of a float (no NaN) as its place in their order, and back.  -0 has +0's place, and neighbouring floats have neighbouring places: a search
// that halves an interval of places always ends.  (Bits with 16 zeros at the end, a bf16 number's, have a place with 16 zeros at the end.)
MQ_HOST_DEVICE uint32_t order_of_bits(uint32_t b) { return b & 0x80000000u ? 0u - b : b | 0x80000000u; }
MQ_HOST_DEVICE uint32_t bits_of_order(uint32_t k) { return k & 0x80000000u ? k ^ 0x80000000u : 0u - k; }

// Place k (0 .. n - 1, downwards) of n that divide [lo, hi) evenly.  Of hi - lo >= 2 the first one lies between, so one of the two bounds moves to
// it or past it.
MQ_HOST_DEVICE uint32_t order_between(uint32_t lo, uint32_t hi, int k, int n) {
  return lo + (uint32_t)((uint64_t)(hi - lo) * (uint32_t)(n - k) / (uint32_t)(n + 1));
}

}  // namespace mq
