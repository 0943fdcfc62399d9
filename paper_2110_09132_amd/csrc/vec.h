// Vectors of consecutive elements in fp32 registers, and sums over groups of
// lanes: what the kernels of the dense operators share.
#pragma once

#include "common.h"

namespace emb {

struct bf16 {
  uint16_t bits;
};

// Accesses of 4, 8 and 16 bytes whose address is a multiple of the element
// size only: rows of odd widths and slices of flat buffers start anywhere, and
// the memory pipeline takes such addresses in one instruction (an access that
// crosses a line costs that line as well, nothing else).
typedef uint32_t words4_f __attribute__((ext_vector_type(4), aligned(4), may_alias));  // 4 fp32
typedef uint32_t words4_h __attribute__((ext_vector_type(4), aligned(2), may_alias));  // 8 bf16
typedef uint32_t words2_h __attribute__((ext_vector_type(2), aligned(2), may_alias));  // 4 bf16

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(bf16 x) { return __uint_as_float(static_cast<uint32_t>(x.bits) << 16); }

// Rounded to nearest even (one instruction for two values); NaN stays NaN.
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ void narrow(float x, float* p) { *p = x; }
__device__ __forceinline__ void narrow(float x, bf16* p) { p->bits = static_cast<uint16_t>(bf16_pair(x, x)); }

// N consecutive elements as they stand in memory; kStream: read with a streaming
// load (data that the call reads once).  load(p, n): only the first n of them are
// read (n may be 0 or less: none), the others are 0.
template <typename T, int N>
struct Vec;
template <int N>
struct Vec<float, N> {
  static_assert(N % 4 == 0, "whole 16-byte words");
  float x[N];
  template <bool kStream = false>
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= N) {
#pragma unroll
      for (int k = 0; k < N / 4; ++k) {
        const words4_f* q = reinterpret_cast<const words4_f*>(p) + k;
        const words4_f w = kStream ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * k + e] = __uint_as_float(w[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = e < n ? p[e] : 0.0f;
    }
  }
  __device__ __forceinline__ float operator[](int e) const { return x[e]; }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < N; ++e) x[e] = 0.0f;
  }
};
template <int N>
struct Vec<bf16, N> {
  static_assert(N == 4 || N % 8 == 0, "whole words");
  uint32_t w[N / 2];
  template <bool kStream = false>
  __device__ __forceinline__ void load(const bf16* p, int n) {
    if (n >= N) {
      if constexpr (N == 4) {
        const words2_h* q = reinterpret_cast<const words2_h*>(p);
        const words2_h v = kStream ? __builtin_nontemporal_load(q) : *q;
        w[0] = v[0];
        w[1] = v[1];
      } else {
#pragma unroll
        for (int k = 0; k < N / 8; ++k) {
          const words4_h* q = reinterpret_cast<const words4_h*>(p) + k;
          const words4_h v = kStream ? __builtin_nontemporal_load(q) : *q;
#pragma unroll
          for (int e = 0; e < 4; ++e) w[4 * k + e] = v[e];
        }
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; e += 2)
        w[e / 2] = (e < n ? p[e].bits : 0u) | (e + 1 < n ? static_cast<uint32_t>(p[e + 1].bits) << 16 : 0u);
    }
  }
  __device__ __forceinline__ float operator[](int e) const {
    return __uint_as_float(e % 2 == 0 ? w[e / 2] << 16 : w[e / 2] & 0xFFFF0000u);
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < N / 2; ++e) w[e] = 0;
  }
};

// v[0 .. N) = p[0 .. N), widened exactly.
template <int N, typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&v)[N]) {
  Vec<T, N> x;
  x.load(p, N);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = x[e];
}

template <bool kStream = false, int N>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[N]) {
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    words4_f w;
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = __float_as_uint(v[4 * k + e]);
    words4_f* q = reinterpret_cast<words4_f*>(p) + k;
    if (kStream)
      __builtin_nontemporal_store(w, q);
    else
      *q = w;
  }
}
template <bool kStream = false, int N>
__device__ __forceinline__ void store_vec(bf16* p, const float (&v)[N]) {
  if constexpr (N == 4) {
    words2_h w;
    w[0] = bf16_pair(v[0], v[1]);
    w[1] = bf16_pair(v[2], v[3]);
    words2_h* q = reinterpret_cast<words2_h*>(p);
    if (kStream)
      __builtin_nontemporal_store(w, q);
    else
      *q = w;
  } else {
#pragma unroll
    for (int k = 0; k < N / 8; ++k) {
      words4_h w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bf16_pair(v[8 * k + 2 * e], v[8 * k + 2 * e + 1]);
      words4_h* q = reinterpret_cast<words4_h*>(p) + k;
      if (kStream)
        __builtin_nontemporal_store(w, q);
      else
        *q = w;
    }
  }
}

// The same for the first n of the N elements only (n may be 0 or less: none); the others read as `fill`.
template <bool kStream = false, int N, typename T>
__device__ __forceinline__ void load_part(const T* p, int n, float fill, float (&v)[N]) {
  Vec<T, N> x;
  x.template load<kStream>(p, n);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = e < n ? x[e] : fill;
}
template <bool kStream = false, int N, typename T>
__device__ __forceinline__ void store_part(T* p, int n, const float (&v)[N]) {
  if (n >= N) {
    store_vec<kStream>(p, v);
    return;
  }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (e < n) narrow(v[e], p + e);
}

// Sum over groups of L consecutive lanes, in every lane of the group, always
// by the same tree: neighbours inside a quad, mirrored halves of 8 and of 16
// lanes, then the rows of 16 and the halves of 32 lanes swapped.
template <int kCtrl>
__device__ __forceinline__ float dpp_read(float x) {
  return __uint_as_float(dpp_move<kCtrl, 0xf>(__float_as_uint(x)));
}
template <int L>
__device__ __forceinline__ float group_sum(float x) {
  static_assert(L == 1 || L == 2 || L == 4 || L == 8 || L == 16 || L == 32 || L == 64, "a power of two");
  if constexpr (L >= 2) x += dpp_read<0xB1>(x);   // quad_perm:[1,0,3,2]
  if constexpr (L >= 4) x += dpp_read<0x4E>(x);   // quad_perm:[2,3,0,1]
  if constexpr (L >= 8) x += dpp_read<0x141>(x);  // row_half_mirror
  if constexpr (L >= 16) x += dpp_read<0x140>(x); // row_mirror
  if constexpr (L >= 32) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  if constexpr (L >= 64) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  }
  return x;
}

}  // namespace emb
