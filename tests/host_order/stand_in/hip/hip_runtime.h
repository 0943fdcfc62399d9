// Stand-in for the HIP headers that lets the host compiler build kernels as ordinary functions, which run on fibers, one
// per lane (fibers.h has the model).  Only what block.hip and its headers name is here.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstring>

#define __global__
#define __device__
#define __host__
#define __forceinline__ inline
#define __shared__ static
#define __launch_bounds__(...)

struct float2 {
  float x, y;
};
struct float4 {
  float x, y, z, w;
};
struct uint2 {
  uint32_t x, y;
};
inline float2 make_float2(float x, float y) { return {x, y}; }
inline uint2 make_uint2(uint32_t x, uint32_t y) { return {x, y}; }
inline float4 make_float4(float x, float y, float z, float w) { return {x, y, z, w}; }
struct dim3 {
  uint32_t x, y, z;
  constexpr dim3(uint32_t x_ = 1, uint32_t y_ = 1, uint32_t z_ = 1) : x(x_), y(y_), z(z_) {}
};
extern dim3 threadIdx, blockIdx, blockDim, gridDim;

typedef int hipError_t;
typedef void* hipStream_t;
typedef void* hipEvent_t;
constexpr hipError_t hipSuccess = 0;
inline hipError_t hipGetLastError() { return hipSuccess; }

using std::max;
using std::min;
inline uint32_t __float_as_uint(float x) { return __builtin_bit_cast(uint32_t, x); }
inline float __uint_as_float(uint32_t x) { return __builtin_bit_cast(float, x); }
inline uint32_t __lane_id() { return threadIdx.x % 64; }

// fibers.h
void __syncthreads();
uint32_t lane_read(uint32_t x, uint32_t from);          // x of lane `from` of the wave
void lane_store(void* p, const void* value, size_t n);  // reaches memory with the stores of the wave's other lanes

// What the headers name beside that; no kernel here calls these.
uint64_t __ballot(bool);
int __popcll(uint64_t);
int32_t atomicOr(int32_t*, int32_t);
int __builtin_amdgcn_readfirstlane(int);
int __builtin_amdgcn_readlane(int, int);
void __builtin_amdgcn_wave_barrier();

inline float __shfl_xor(float x, int mask, int = 64) {
  return __uint_as_float(lane_read(__float_as_uint(x), __lane_id() ^ static_cast<uint32_t>(mask)));
}
// the moves of group_sum: quad_perm:[1,0,3,2] and [2,3,0,1], row_half_mirror, row_mirror
inline int __builtin_amdgcn_update_dpp(int, int x, int ctrl, int, int, bool) {
  const uint32_t l = __lane_id();
  const uint32_t from = ctrl == 0xB1 ? l ^ 1 : ctrl == 0x4E ? l ^ 2 : ctrl == 0x141 ? l ^ 7 : l ^ 15;
  return static_cast<int>(lane_read(static_cast<uint32_t>(x), from));
}
struct Swapped {
  uint32_t r[2];
  uint32_t operator[](int i) const { return r[i]; }
};
inline Swapped swapped(uint32_t x, uint32_t bit) {
  const uint32_t l = __lane_id(), other = lane_read(x, l ^ bit);
  return l & bit ? Swapped{{other, x}} : Swapped{{x, other}};
}
inline Swapped __builtin_amdgcn_permlane16_swap(uint32_t x, uint32_t, bool, bool) { return swapped(x, 16); }
inline Swapped __builtin_amdgcn_permlane32_swap(uint32_t x, uint32_t, bool, bool) { return swapped(x, 32); }

template <typename V, typename P>
inline void store_whole(const V& v, P* p) {
  lane_store(p, &v, sizeof(v));
}
#define __builtin_nontemporal_store(v, p) store_whole(v, p)
