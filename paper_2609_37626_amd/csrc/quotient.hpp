// The quotient that a cache's code is rounded from (host and device).
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>

namespace splash {

// y / scale as a division gives it, by scale's inverse: their product and one correction.
// scale >= 2^-100, below which what is left over would pass fp32's range; from 2^-90 on, and
// for quotients from 2^-11 on, the bits are the division's, else the codes.  (A host test
// compares them over all of scale's fractions, at and beside the ties of E4M3.)
template <bool FINITE>
__host__ __device__ __forceinline__ float quotient(float y, float scale, float inverse) {
  const float q = y * inverse;
  const float r = copysignf(__builtin_fmaf(__builtin_fmaf(-q, scale, y), inverse, q), y);
  return FINITE || fabsf(q) < 1e30f ? r : q;
}

}  // namespace splash
