// How the kernels of layer norm and of the norms around a block spread rows over
// lanes, and their row sums.
#pragma once

#include <type_traits>

#include "vec.h"

namespace emb {

// How a row of D elements is spread: kE elements per lane and vector.  A row
// that `narrow` elements per lane hold takes one wave, or `lanes` lanes of one
// (several rows per wave; one lane where it is no whole vector); wider rows take
// 2, 4 or 8 waves, those of 8 up to kMaxElems elements per lane; the widest are
// read again from memory for every pass over them.  With kMaxElems per lane two
// waves are left out (forward, 8192 x 4096 fp32: 70 us with two waves per row,
// 49 us with four).
constexpr int kMaxElems = 32;
struct RowPlan {
  int waves;  // waves per row: 1, 2, 4, 8; 0: the row does not fit registers
  int lanes;  // lanes per row where waves == 1
  int nv;     // vectors per lane
};
constexpr RowPlan plan_row(int D, int E, int narrow) {
  const int nvec = (D + E - 1) / E;
  if (D < E) return {1, 1, 1};
  if (nvec <= kWave) {
    int l = 8;
    while (l < nvec) l *= 2;
    return {1, l, 1};
  }
  for (const int w : {1, 2, 4, 8}) {
    if (w == 2 && narrow == kMaxElems) continue;
    const int nv = (nvec + w * kWave - 1) / (w * kWave);
    if (nv * E <= (w < 8 ? narrow : kMaxElems)) return {w, kWave, nv <= 4 ? nv : nv <= 6 ? 6 : 8};
  }
  return {0, kWave, 0};
}

// The columns of a lane's vectors.  The vector that the row's end cuts is moved
// back so that it ends there, as are those past the end: every load is a whole
// vector, without a branch (65536 x 1023 bf16: 83 us with element loads at the
// rows' ends, 53 us so, 47 us for 1024; backward 184, 87 and 77 us), and the
// elements that a vector shares with the ones before it are left out of sums
// (where they are stored, the same value is stored twice).  plan_row leaves such
// vectors in the last place of a lane, or in the last two.  kLanes == 1: the row
// is a part of one vector.
template <int kE, int kLanes, int kNV>
struct Columns {
  int lane, D;
  static constexpr bool kPart = kLanes == 1;
  __device__ __forceinline__ static constexpr bool ends(int k) { return k >= kNV - (kNV > 4 ? 2 : 1); }
  __device__ __forceinline__ int first(int k) const {
    const int c = (k * kLanes + lane) * kE;
    return ends(k) && !kPart ? min(c, D - kE) : c;
  }
  // Elements at the front of vector k that belong to others (kE or more: all).
  __device__ __forceinline__ int shared(int k) const {
    return ends(k) && !kPart ? (k * kLanes + lane) * kE - first(k) : 0;
  }
  __device__ __forceinline__ bool own(int k, int e) const {
    return kPart ? e < D : ends(k) ? e >= shared(k) : true;
  }
  template <bool kStream, typename T>
  __device__ __forceinline__ void load(const T* row, int k, Vec<T, kE>& v) const {
    v.template load<kStream>(row + first(k), kPart ? D : kE);
  }
  __device__ __forceinline__ void load(const float* row, int k, float fill, float (&v)[kE]) const {
    load_part(row + first(k), row == nullptr ? 0 : kPart ? D : kE, fill, v);
  }
  template <bool kStream, typename T>
  __device__ __forceinline__ void store(T* row, int k, const float (&v)[kE]) const {
    if (kPart)
      store_part(row, D, v);
    else if (shared(k) < kE)
      store_vec<kStream>(row + first(k), v);
  }
};

// Sum over a row's lanes, in all of them.  kW > 1: through LDS, in wave order;
// `slot` alternates so that one barrier per sum is enough.
template <int kL, int kW>
__device__ __forceinline__ float row_sum(float x, float (*red)[kW > 1 ? kW : 1], int slot) {
  x = group_sum<(kW > 1 ? kWave : kL)>(x);
  if constexpr (kW > 1) {
    if (lane_id() == 0) red[slot][threadIdx.x / kWave] = x;
    __syncthreads();
    x = red[slot][0];
#pragma unroll
    for (int w = 1; w < kW; ++w) x += red[slot][w];
  }
  return x;
}
// Two sums at once; a workgroup of kWaves waves may hold several rows of kW waves.
template <int kL, int kW, int kWaves>
__device__ __forceinline__ void row_sum2(float& a, float& b, float2 (*red)[kWaves], int slot) {
  a = group_sum<(kW > 1 ? kWave : kL)>(a);
  b = group_sum<(kW > 1 ? kWave : kL)>(b);
  if constexpr (kW > 1) {
    const int wave = static_cast<int>(threadIdx.x) / kWave;
    if (lane_id() == 0) red[slot][wave] = make_float2(a, b);
    __syncthreads();
    const float2* r = red[slot] + wave / kW * kW;
    a = r[0].x;
    b = r[0].y;
#pragma unroll
    for (int w = 1; w < kW; ++w) {
      a += r[w].x;
      b += r[w].y;
    }
  }
}

// Whether any row of more than one vector per lane is planned with this shape.
template <int kE, int kNarrow>
constexpr bool planned(int waves, int nv) {
  for (int D = kWave * kE + kE; D <= 8 * kWave * kMaxElems; D += kE) {
    const RowPlan pl = plan_row(D, kE, kNarrow);
    if (pl.waves == waves && pl.nv == nv) return true;
  }
  return false;
}
// Calls f(L, NV, W) with the shape of plan_row(D, kE, kNarrow) as integral constants.
template <int N>
using Int = std::integral_constant<int, N>;
template <int kE, int kNarrow, typename F>
void with_shape(const RowPlan& pl, F&& f) {
  if (pl.waves == 1 && pl.nv == 1) {
    switch (pl.lanes) {
      case 1: return f(Int<1>{}, Int<1>{}, Int<1>{});
      case 8: return f(Int<8>{}, Int<1>{}, Int<1>{});
      case 16: return f(Int<16>{}, Int<1>{}, Int<1>{});
      case 32: return f(Int<32>{}, Int<1>{}, Int<1>{});
      default: return f(Int<64>{}, Int<1>{}, Int<1>{});
    }
  }
  const auto shape = [&](auto W, auto NV) {
    if constexpr (planned<kE, kNarrow>(W.value, NV.value))
      if (pl.waves == W.value && pl.nv == NV.value) f(Int<64>{}, NV, W);
  };
  const auto shapes = [&](auto W) {  // every nv that plan_row gives
    static_assert(kMaxElems / kE <= 8, "up to 8 vectors per lane");
    shape(W, Int<1>{});
    shape(W, Int<2>{});
    shape(W, Int<3>{});
    shape(W, Int<4>{});
    shape(W, Int<6>{});
    shape(W, Int<8>{});
  };
  shapes(Int<1>{});
  shapes(Int<2>{});
  shapes(Int<4>{});
  shapes(Int<8>{});
}

}  // namespace emb
