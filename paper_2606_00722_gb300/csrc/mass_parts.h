// Masses of a histogram's bins in two 32-bit sums, and where a running total
// passes a target.  Plain C++: the kernels and the host's tests include it.
#pragma once
#include <stdint.h>

#ifdef __CUDACC__
#define EPIC_INLINE __host__ __device__ __forceinline__
#else
#define EPIC_INLINE inline
#endif

namespace epic {

// Most elements of a slice whose masses, in these parts, a histogram's 32-bit bins can add up.
constexpr int kSliceElems = 131000;

// An element's mass, at most 2^30, is low + 2^15 high with low within 2^14 of 0 and high at most 2^15.  So the sums over a
// slice of at most kSliceElems elements fit 32 bits: high's an unsigned one (131,000 2^15 < 2^32), low's a signed one
// (131,000 2^14 < 2^31).  A low part from 0 up to 2^15 would pass 2^31 from 65,539 elements on.
struct MassParts {
  uint32_t high, low;  // low: the bits of a signed number
  EPIC_INLINE uint64_t value() const { return ((uint64_t)high << 15) + (uint64_t)(int64_t)(int32_t)low; }
};

EPIC_INLINE MassParts mass_parts(uint32_t mass) {
  const uint32_t high = (mass + (1u << 14)) >> 15;
  return {high, mass - (high << 15)};
}

// Whether the running total passes t at an element of mass q with `before` ahead of it; the last one takes what lies past
// the end, so of a list's elements exactly one answers, whatever t is.
EPIC_INLINE bool passes(uint64_t before, uint64_t q, uint64_t t, bool last) {
  return before <= t && (t - before < q || last);
}

}  // namespace epic
