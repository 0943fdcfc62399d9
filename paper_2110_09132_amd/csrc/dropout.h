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

// v[e] = scale v[e] where element (t, c + e) is kept, 0 elsewhere; c is a multiple of 4, per = ceil(D / 4).
template <int N>
__device__ __forceinline__ void apply_mask(const DropMask& m, uint64_t key, int64_t t, int64_t per, int c, float (&v)[N]) {
  static_assert(N % 4 == 0, "whole draws");
#pragma unroll
  for (int k = 0; k < N / 4; ++k) {
    const uint64_t r = mask_draw(key, t * per + c / 4 + k);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * k + e] = kept(r, e, m.cut) ? v[4 * k + e] * m.scale : 0.0f;
  }
}

}  // namespace emb
