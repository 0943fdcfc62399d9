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

// The bits of elements 4 j .. 4 j + 3 of row t, where n = t ceil(D / 4) + j.
__device__ __forceinline__ uint64_t mask_draw(uint64_t key, int64_t n) {
  return mix64(key + static_cast<uint64_t>(n + 1) * kGamma);
}
__device__ __forceinline__ bool kept(uint64_t draw, int e, uint32_t cut) {
  return (static_cast<uint32_t>(draw >> (16 * e)) & 0xFFFFu) >= cut;
}

// Bit e: element (t, c + e) is kept; per = ceil(D / 4).  Where c is no multiple of 4 the bits come from one draw more.
template <int N>
__device__ __forceinline__ uint32_t mask_bits(const DropMask& m, uint64_t key, int64_t t, int64_t per, int c) {
  static_assert(N % 4 == 0, "whole draws");
  const int64_t n = t * per + c / 4;
  const int odd = c % 4;
  uint64_t r[N / 4];
#pragma unroll
  for (int k = 0; k < N / 4; ++k) r[k] = mask_draw(key, n + k);
  if (odd != 0) {
    const uint64_t last = mask_draw(key, n + N / 4);
#pragma unroll
    for (int k = 0; k < N / 4; ++k) r[k] = r[k] >> (16 * odd) | (k + 1 < N / 4 ? r[k + 1] : last) << (64 - 16 * odd);
  }
  uint32_t bits = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) bits |= kept(r[e / 4], e % 4, m.cut) ? 1u << e : 0u;
  return bits;
}

// v[e] = scale v[e] where element (t, c + e) is kept, 0 elsewhere.
template <int N>
__device__ __forceinline__ void apply_mask(const DropMask& m, uint64_t key, int64_t t, int64_t per, int c, float (&v)[N]) {
  const uint32_t bits = mask_bits<N>(m, key, t, per, c);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = bits >> e & 1u ? v[e] * m.scale : 0.0f;
}

}  // namespace emb
