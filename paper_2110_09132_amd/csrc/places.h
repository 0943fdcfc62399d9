// Places in the map of the relative position bias's buckets (bias.hip).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace emb {

// Place in bucket_of [2 R + 1] of the difference `first` + u, for 0 <= u < 2^30
// and R < 2^30, in 32 bits: place(base_of(first, R), u, R).  2 R + u does not
// fit them, so the upper end is taken off before u is added.
__host__ __device__ __forceinline__ int32_t base_of(int64_t first, int32_t R) {
  const int64_t b = first + R, low = -(1 << 30), high = 2 * static_cast<int64_t>(R);
  return static_cast<int32_t>(b < low ? low : b > high ? high : b);
}
__host__ __device__ __forceinline__ int32_t place(int32_t base, int32_t u, int32_t R) {
  const int32_t last = 2 * R - u;
  const int32_t p = (base < last ? base : last) + u;
  return p < 0 ? 0 : p;
}

}  // namespace emb
