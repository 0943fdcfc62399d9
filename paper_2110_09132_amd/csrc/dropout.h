// The mask of emb_dropout: 16 random bits per element, four elements of a row per draw.
#pragma once

#include "common.h"
#include "launch.h"

namespace emb {

constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

// SplitMix64's output function (Steele, Lea & Flood 2014).
__host__ __device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}

__device__ __forceinline__ uint64_t mask_key(const DropMask& m) {
  return m.seed_dev != nullptr ? mix64(*m.seed_dev) : m.key;
}

// The generator's state before it is mixed, for elements 4 j .. 4 j + 3 of row t: n = t ceil(D / 4) + j.  The next four
// elements' is kGamma more, so a row's states follow from one multiplication.
__device__ __forceinline__ uint64_t mask_state(uint64_t key, int64_t n) { return key + static_cast<uint64_t>(n + 1) * kGamma; }

// keep[e]: element c + e of the row is kept, where `state` is that of element 4 (c / 4).  Where c is no multiple of 4
// (odd = c % 4) the bits come from one draw more.
template <int N>
__device__ __forceinline__ void mask_bits(uint32_t cut, uint64_t state, int odd, bool (&keep)[N]) {
  static_assert(N % 4 == 0, "whole draws");
  uint64_t r[N / 4];
#pragma unroll
  for (int k = 0; k < N / 4; ++k) r[k] = mix64(state + k * kGamma);
  if (odd != 0) {
    const uint64_t last = mix64(state + N / 4 * kGamma);
#pragma unroll
    for (int k = 0; k < N / 4; ++k) r[k] = r[k] >> (16 * odd) | (k + 1 < N / 4 ? r[k + 1] : last) << (64 - 16 * odd);
  }
#pragma unroll
  for (int e = 0; e < N; ++e) {  // 16 bits at the top of a word against the cut at the top of a word
    const uint32_t w = static_cast<uint32_t>(r[e / 4] >> (32 * (e / 2 % 2)));
    keep[e] = (e % 2 == 0 ? w << 16 : w) >= cut << 16;
  }
}

// v[e] = scale v[e] where element (t, c + e) is kept, 0 elsewhere; per = ceil(D / 4).
template <int N>
__device__ __forceinline__ void apply_mask(const DropMask& m, uint64_t key, int64_t t, int64_t per, int c, float (&v)[N]) {
  bool keep[N];
  mask_bits(m.cut, mask_state(key, t * per + c / 4), c % 4, keep);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = keep[e] ? v[e] * m.scale : 0.0f;
}

}  // namespace emb
