// Bins of equal width, from the largest of some numbers down to the smallest.
#pragma once
#include <hip/hip_runtime.h>

#include <cfloat>
#include <cmath>

namespace {

// Bins a unit, with which (int)((top - v) * scale) is one of `bins` for every v that `span` (finite) reaches.  Where numbers differ by next to nothing, less than 7.5e-37 with
// 256 bins, the quotient is beyond fp32: times a difference it would be infinite, or no number, and its whole part no bin.
__host__ __device__ __forceinline__ float bin_scale(int bins, float span) { return span > 0.f ? fminf((float)(bins - 1) / span, FLT_MAX) : 0.f; }
// a number that none in bins 0 .. b is below, by the arithmetic that puts them there
__host__ __device__ __forceinline__ float bin_edge(int b, float top, float scale) {
  if (scale == 0.f) return top;
  const float e = top - (float)(b + 1) / scale;
  return e - (4e-7f * (fabsf(top) + fabsf(e)) + 1e-37f);
}

}  // namespace
