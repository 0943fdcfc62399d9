// Layer norm of rows, forward and backward.
//
//   mean = sum x / D;  rstd = 1 / sqrt(sum (x - mean)^2 / D + eps);  xh = (x - mean) rstd
//   y  = xh w + b
//   dx = rstd (g - c1 - xh c2),  g = dy w,  c1 = sum g / D,  c2 = sum g xh / D
//   dw = sum over rows of dy xh,  db = sum over rows of dy
//
// Both directions are bound by memory: the row is read once and stays in
// registers (kE consecutive elements per lane and vector, kNV vectors), so the
// variance is summed from the differences to the mean and not from squares.
// Rows come from x directly, or from a table by id: the lookup then costs no
// pass of its own.  Statistics and sums are fp32.
#include <type_traits>

#include "vec.h"
#include "launch.h"

namespace emb {
namespace {

// How a row of D elements is spread: kE elements per lane and vector; up to
// kMaxElems elements of a row per lane.  Rows that one wave can hold take
// `lanes` lanes (several rows per wave for narrow ones); wider rows take 4 or
// 8 waves; the widest are read again from memory for every pass over them.
constexpr int kMaxElems = 32;
constexpr int kThreads = 256;
struct RowPlan {
  int waves;  // waves per row: 1, 4, 8; 0: the row does not fit registers
  int lanes;  // lanes per row where waves == 1
  int nv;     // vectors per lane
};
RowPlan plan_row(int D, int E) {
  const int nvec = (D + E - 1) / E;
  const int most = kMaxElems / E;
  if (nvec <= kWave) {
    int l = 8;
    while (l < nvec) l *= 2;
    return {1, l, 1};
  }
  const auto round_nv = [](int nv) { return nv <= 4 ? nv : nv <= 6 ? 6 : 8; };
  for (const int w : {1, 4, 8}) {
    const int nv = (nvec + w * kWave - 1) / (w * kWave);
    if (nv <= most) return {w, kWave, round_nv(nv)};
  }
  return {0, kWave, 0};
}

template <typename T>
struct Rows {
  T* p;
  int64_t ld;
};

// Source row of row t: t itself, or ids[t]; an id outside [0, V) reads as a row of zeros.
template <typename XT>
struct Source {
  const XT* p;
  int64_t ld;
  const int32_t* ids;
  int64_t V;
  __device__ __forceinline__ const XT* row(int64_t t, bool& bad) const {
    if (ids == nullptr) return p + t * ld;
    const int32_t id = ids[t];
    if (id < 0 || id >= V) {
      bad = true;
      return nullptr;
    }
    return p + id * ld;
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
// Two sums at once.
template <int kL, int kW>
__device__ __forceinline__ void row_sum2(float& a, float& b, float (*red)[kW > 1 ? 2 * kW : 1], int slot) {
  a = group_sum<(kW > 1 ? kWave : kL)>(a);
  b = group_sum<(kW > 1 ? kWave : kL)>(b);
  if constexpr (kW > 1) {
    if (lane_id() == 0) {
      red[slot][threadIdx.x / kWave] = a;
      red[slot][kW + threadIdx.x / kWave] = b;
    }
    __syncthreads();
    a = red[slot][0];
    b = red[slot][kW];
#pragma unroll
    for (int w = 1; w < kW; ++w) {
      a += red[slot][w];
      b += red[slot][kW + w];
    }
  }
}

template <typename XT, typename YT, int kE, int kL, int kNV, int kW>
__global__ __launch_bounds__(kW > 4 ? kW * kWave : kThreads) void norm_kernel(
    Source<XT> src, int64_t T, int D, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
    Rows<YT> y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int32_t* status) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kRows = (kW > 4 ? kW * kWave : kThreads) / kLanes;
  __shared__ float red[2][kW > 1 ? kW : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  const int sub = static_cast<int>(threadIdx.x) / kLanes;
  const float fD = static_cast<float>(D);
  bool bad = false;
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows; t0 < T; t0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t t = t0 + sub;
    const XT* row = t < T ? src.row(t, bad) : nullptr;
    float v[kNV][kE];
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      const int c = (k * kLanes + lane) * kE;
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, v[k]);
#pragma unroll
      for (int e = 0; e < kE; ++e) s += v[k][e];
    }
    const float mean = row_sum<kL, kW>(s, red, 0) / fD;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      const int c = (k * kLanes + lane) * kE;
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        v[k][e] = c + e < D ? v[k][e] - mean : 0.0f;
        s += v[k][e] * v[k][e];
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<kL, kW>(s, red, 1) / fD + eps);
    if (t < T) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        const int c = (k * kLanes + lane) * kE;
        float w[kE], b[kE];
        load_part(weight + c, weight != nullptr ? D - c : 0, 1.0f, w);
        load_part(bias + c, bias != nullptr ? D - c : 0, 0.0f, b);
#pragma unroll
        for (int e = 0; e < kE; ++e) v[k][e] = v[k][e] * rstd * w[e] + b[e];
        store_part(y.p + t * y.ld + c, D - c, v[k]);
      }
      if (lane == 0) {
        mean_out[t] = mean;
        rstd_out[t] = rstd;
      }
    }
  }
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
}

// Rows too wide for registers: one workgroup per row, which reads the row
// three times (the second and third time from the caches).
constexpr int kLoopWaves = 16;
template <typename XT, typename YT>
__global__ __launch_bounds__(kLoopWaves* kWave) void norm_loop_kernel(
    Source<XT> src, int64_t T, int D, const float* __restrict__ weight, const float* __restrict__ bias, float eps,
    Rows<YT> y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int32_t* status) {
  constexpr int kStep = kLoopWaves * kWave * 4;
  __shared__ float red[2][kLoopWaves];
  const float fD = static_cast<float>(D);
  bool bad = false;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const XT* row = src.row(t, bad);
    float v[4], s = 0.0f;
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += kStep) {
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, v);
      s += (v[0] + v[1]) + (v[2] + v[3]);
    }
    const float mean = row_sum<kWave, kLoopWaves>(s, red, 0) / fD;
    s = 0.0f;
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += kStep) {
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, v);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float d = c + e < D ? v[e] - mean : 0.0f;
        s += d * d;
      }
    }
    const float rstd = 1.0f / sqrtf(row_sum<kWave, kLoopWaves>(s, red, 1) / fD + eps);
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += kStep) {
      float w[4], b[4];
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, v);
      load_part(weight + c, weight != nullptr ? D - c : 0, 1.0f, w);
      load_part(bias + c, bias != nullptr ? D - c : 0, 0.0f, b);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (v[e] - mean) * rstd * w[e] + b[e];
      store_part(y.p + t * y.ld + c, D - c, v);
    }
    if (threadIdx.x == 0) {
      mean_out[t] = mean;
      rstd_out[t] = rstd;
    }
  }
  if (bad && threadIdx.x == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
}

// The backward pass.  A workgroup takes every gridDim.x-th group of rows and
// keeps its columns' sums for dw and db in registers; at the end the rows that
// share a workgroup are joined (lanes, then waves through LDS) into one partial
// row of the workspace, [gridDim.x][2][D], which norm_sum_kernel adds up in
// workgroup order: the result depends on the sizes only, not on timing.
template <typename XT, typename GT, int kE, int kL, int kNV, int kW>
__global__ __launch_bounds__(kW > 4 ? kW * kWave : kThreads) void norm_grad_kernel(
    Rows<const GT> dy, Source<XT> src, int64_t T, int D, const float* __restrict__ weight,
    const float* __restrict__ mean_in, const float* __restrict__ rstd_in, Rows<GT> dx, float* __restrict__ part,
    int32_t* status) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kRows = (kW > 4 ? kW * kWave : kThreads) / kLanes;
  constexpr int kWaves = kW > 1 ? 1 : kThreads / kWave;  // waves that hold sums of the same columns
  __shared__ float red[2][kW > 1 ? 2 * kW : 1];
  __shared__ float join[kWaves > 1 ? kWaves : 1][kWaves > 1 ? kLanes * kNV * kE : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  const int sub = static_cast<int>(threadIdx.x) / kLanes;
  const float fD = static_cast<float>(D);
  bool bad = false;
  float dw[kNV][kE] = {}, db[kNV][kE] = {};
  int slot = 0;
  for (int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows; t0 < T; t0 += static_cast<int64_t>(gridDim.x) * kRows) {
    const int64_t t = t0 + sub;
    const bool live = t < T;
    const XT* row = live ? src.row(t, bad) : nullptr;
    const GT* grow = dy.p + t * dy.ld;
    const float mean = live ? mean_in[t] : 0.0f, rstd = live ? rstd_in[t] : 0.0f;
    float xh[kNV][kE], g[kNV][kE];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      const int c = (k * kLanes + lane) * kE;
      float w[kE];
      load_part(row + c, row != nullptr ? D - c : 0, row != nullptr ? mean : 0.0f, xh[k]);
      load_part(grow + c, live ? D - c : 0, 0.0f, g[k]);
      load_part(weight + c, weight != nullptr ? D - c : 0, 1.0f, w);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        xh[k][e] = (xh[k][e] - mean) * rstd;
        dw[k][e] += g[k][e] * xh[k][e];
        db[k][e] += g[k][e];
        g[k][e] *= w[e];
        s1 += g[k][e];
        s2 += g[k][e] * xh[k][e];
      }
    }
    row_sum2<kL, kW>(s1, s2, red, slot);
    slot ^= 1;
    const float c1 = s1 / fD, c2 = s2 / fD;
    if (live && dx.p != nullptr) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        const int c = (k * kLanes + lane) * kE;
#pragma unroll
        for (int e = 0; e < kE; ++e) g[k][e] = rstd * (g[k][e] - c1 - xh[k][e] * c2);
        store_part(dx.p + t * dx.ld + c, D - c, g[k]);
      }
    }
  }
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
  if (part == nullptr) return;
  float* out = part + static_cast<size_t>(blockIdx.x) * 2 * D;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float(&a)[kNV][kE] = which == 0 ? dw : db;
    if constexpr (kL < kWave) {  // the rows of a wave
#pragma unroll
      for (int k = 0; k < kNV; ++k)
#pragma unroll
        for (int e = 0; e < kE; ++e)
          for (int m = kL; m < kWave; m *= 2) a[k][e] += __shfl_xor(a[k][e], m, kWave);
    }
    if constexpr (kWaves > 1) {  // the waves of the workgroup
      const int w = static_cast<int>(threadIdx.x) / kWave;
      if (static_cast<int>(lane_id()) < kLanes) {
#pragma unroll
        for (int k = 0; k < kNV; ++k)
#pragma unroll
          for (int e = 0; e < kE; ++e) join[w][(k * kLanes + lane) * kE + e] = a[k][e];
      }
      __syncthreads();
      for (int c = static_cast<int>(threadIdx.x); c < D; c += kThreads) {
        float s = join[0][c];
#pragma unroll
        for (int i = 1; i < kWaves; ++i) s += join[i][c];
        out[static_cast<size_t>(which) * D + c] = s;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        const int c = (k * kLanes + lane) * kE;
        store_part(out + static_cast<size_t>(which) * D + c, D - c, a[k]);
      }
    }
  }
}

// Rows too wide for registers: dx with one workgroup per row, then the column
// sums with one workgroup per tile of columns and every gridDim.y-th row.
template <typename XT, typename GT>
__global__ __launch_bounds__(kLoopWaves* kWave) void norm_grad_loop_kernel(
    Rows<const GT> dy, Source<XT> src, int64_t T, int D, const float* __restrict__ weight,
    const float* __restrict__ mean_in, const float* __restrict__ rstd_in, Rows<GT> dx, int32_t* status) {
  constexpr int kStep = kLoopWaves * kWave * 4;
  __shared__ float red[2][2 * kLoopWaves];
  const float fD = static_cast<float>(D);
  bool bad = false;
  int slot = 0;
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    const XT* row = src.row(t, bad);
    const GT* grow = dy.p + t * dy.ld;
    const float mean = mean_in[t], rstd = rstd_in[t];
    float x[4], g[4], w[4], s1 = 0.0f, s2 = 0.0f;
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += kStep) {
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, x);
      load_part(grow + c, D - c, 0.0f, g);
      load_part(weight + c, weight != nullptr ? D - c : 0, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s1 += g[e] * w[e];
        s2 += c + e < D ? g[e] * w[e] * ((x[e] - mean) * rstd) : 0.0f;
      }
    }
    row_sum2<kWave, kLoopWaves>(s1, s2, red, slot);
    slot ^= 1;
    const float c1 = s1 / fD, c2 = s2 / fD;
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += kStep) {
      load_part(row + c, row != nullptr ? D - c : 0, 0.0f, x);
      load_part(grow + c, D - c, 0.0f, g);
      load_part(weight + c, weight != nullptr ? D - c : 0, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = rstd * (g[e] * w[e] - c1 - (x[e] - mean) * rstd * c2);
      store_part(dx.p + t * dx.ld + c, D - c, x);
    }
  }
  if (bad && threadIdx.x == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
}

template <typename XT, typename GT>
__global__ __launch_bounds__(kThreads) void norm_columns_kernel(Rows<const GT> dy, Source<XT> src, int64_t T, int D,
                                                                const float* __restrict__ mean_in,
                                                                const float* __restrict__ rstd_in,
                                                                float* __restrict__ part, int32_t* status) {
  const int c = (static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x)) * 4;
  float dw[4] = {}, db[4] = {};
  bool bad = false;
  for (int64_t t = blockIdx.y; t < T; t += gridDim.y) {
    const XT* row = src.row(t, bad);
    float x[4], g[4];
    load_part(row + c, row != nullptr ? D - c : 0, 0.0f, x);
    load_part(dy.p + t * dy.ld + c, D - c, 0.0f, g);
    const float mean = mean_in[t], rstd = rstd_in[t];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dw[e] += c + e < D ? g[e] * ((x[e] - mean) * rstd) : 0.0f;
      db[e] += g[e];
    }
  }
  float* out = part + static_cast<size_t>(blockIdx.y) * 2 * D;
  store_part(out + c, D - c, dw);
  store_part(out + static_cast<size_t>(D) + c, D - c, db);
  if (bad && threadIdx.x == 0) raise_flag(status, EMB_DEV_ID_OUT_OF_RANGE);
}

// out[c] = sum over the nparts partial rows of part[p][c], c < n: a workgroup
// takes kSumCols columns, its lanes' groups every kSumGroups-th partial row.
constexpr int kSumCols = 32;
constexpr int kSumGroups = 32;
__global__ __launch_bounds__(kSumCols* kSumGroups) void norm_sum_kernel(const float* __restrict__ part, int nparts,
                                                                        int D, float* __restrict__ dw,
                                                                        float* __restrict__ db) {
  __shared__ float red[kSumGroups][kSumCols + 1];
  const int col = static_cast<int>(threadIdx.x) % kSumCols, g = static_cast<int>(threadIdx.x) / kSumCols;
  const int64_t c = static_cast<int64_t>(blockIdx.x) * kSumCols + col;
  const int64_t n = 2 * static_cast<int64_t>(D);
  float s = 0.0f;
  if (c < n) {
#pragma unroll 8
    for (int p = g; p < nparts; p += kSumGroups) s += part[p * n + c];
  }
  red[g][col] = s;
  __syncthreads();
  if (g == 0 && c < n) {
#pragma unroll
    for (int i = 1; i < kSumGroups; ++i) s += red[i][col];
    float* out = c < D ? dw : db;
    if (out != nullptr) out[c < D ? c : c - D] = s;
  }
}

// Workgroups of the backward pass, and so the number of partial rows.
constexpr int kGradBlocks = 512;
int grad_blocks(int64_t T, int rows_per_block) {
  const int64_t b = (T + rows_per_block - 1) / rows_per_block;
  return static_cast<int>(b < kGradBlocks ? b : kGradBlocks);
}
int rows_per_block(const RowPlan& pl) { return pl.waves == 1 ? kThreads / pl.lanes : 1; }

// Calls f with the compile-time shape of the plan: f(E, L, NV, W as integral constants).
template <int N>
using Int = std::integral_constant<int, N>;
template <int kE, typename F>
void with_shape(const RowPlan& pl, F&& f) {
  if (pl.waves == 1 && pl.nv == 1) {
    switch (pl.lanes) {
      case 8: return f(Int<8>{}, Int<1>{}, Int<1>{});
      case 16: return f(Int<16>{}, Int<1>{}, Int<1>{});
      case 32: return f(Int<32>{}, Int<1>{}, Int<1>{});
      default: return f(Int<64>{}, Int<1>{}, Int<1>{});
    }
  }
#define EMB_SHAPE(W, NV) \
  if (pl.waves == W && pl.nv == NV) return f(Int<64>{}, Int<NV>{}, Int<W>{})
  EMB_SHAPE(1, 2);
  EMB_SHAPE(1, 3);
  EMB_SHAPE(1, 4);
  EMB_SHAPE(4, 2);
  EMB_SHAPE(4, 3);
  EMB_SHAPE(4, 4);
  EMB_SHAPE(8, 3);
  EMB_SHAPE(8, 4);
  if constexpr (kE == 4) {
    EMB_SHAPE(1, 6);
    EMB_SHAPE(1, 8);
    EMB_SHAPE(4, 6);
    EMB_SHAPE(4, 8);
    EMB_SHAPE(8, 6);
    EMB_SHAPE(8, 8);
  }
#undef EMB_SHAPE
}

template <typename XT, typename YT>
void norm_call(const NormArgs& a, hipStream_t stream) {
  constexpr int kE = std::is_same<XT, bf16>::value && std::is_same<YT, bf16>::value ? 8 : 4;
  const Source<XT> src{static_cast<const XT*>(a.x), a.ldx, a.ids, a.V};
  const Rows<YT> y{static_cast<YT*>(a.y), a.ldy};
  const RowPlan pl = plan_row(a.D, kE);
  const float eps = static_cast<float>(a.eps);
  if (pl.waves == 0) {
    norm_loop_kernel<XT, YT><<<grid_for(a.T, kMaxBlocks), kLoopWaves * kWave, 0, stream>>>(
        src, a.T, a.D, a.weight, a.bias, eps, y, a.mean, a.rstd, a.status);
    return;
  }
  const int rows = rows_per_block(pl);
  const unsigned grid = grid_for((a.T + rows - 1) / rows, kMaxBlocks);
  with_shape<kE>(pl, [&](auto L, auto NV, auto W) {
    norm_kernel<XT, YT, kE, L.value, NV.value, W.value>
        <<<grid, W.value > 4 ? W.value * kWave : kThreads, 0, stream>>>(src, a.T, a.D, a.weight, a.bias, eps, y,
                                                                         a.mean, a.rstd, a.status);
  });
}

template <typename XT, typename GT>
void norm_grad_call(const NormGradArgs& a, hipStream_t stream) {
  constexpr int kE = std::is_same<XT, bf16>::value && std::is_same<GT, bf16>::value ? 8 : 4;
  const Source<XT> src{static_cast<const XT*>(a.x), a.ldx, a.ids, a.V};
  const Rows<const GT> dy{static_cast<const GT*>(a.dy), a.lddy};
  const Rows<GT> dx{static_cast<GT*>(a.dx), a.lddx};
  const bool params = a.dweight != nullptr || a.dbias != nullptr;
  float* part = params ? static_cast<float*>(a.workspace) : nullptr;
  const RowPlan pl = plan_row(a.D, kE);
  int nparts = 0;
  if (a.T > 0 && pl.waves == 0) {
    if (params) {  // first: dx may be written over dy
      nparts = grad_blocks(a.T, 16);
      norm_columns_kernel<XT, GT><<<dim3((a.D + 4 * kThreads - 1) / (4 * kThreads), nparts), kThreads, 0, stream>>>(
          dy, src, a.T, a.D, a.mean, a.rstd, part, a.status);
    }
    if (a.dx != nullptr)
      norm_grad_loop_kernel<XT, GT><<<grid_for(a.T, kMaxBlocks), kLoopWaves * kWave, 0, stream>>>(
          dy, src, a.T, a.D, a.weight, a.mean, a.rstd, dx, a.status);
  } else if (a.T > 0) {
    nparts = grad_blocks(a.T, rows_per_block(pl));
    with_shape<kE>(pl, [&](auto L, auto NV, auto W) {
      norm_grad_kernel<XT, GT, kE, L.value, NV.value, W.value>
          <<<nparts, W.value > 4 ? W.value * kWave : kThreads, 0, stream>>>(dy, src, a.T, a.D, a.weight, a.mean,
                                                                             a.rstd, dx, part, a.status);
    });
  }
  if (params) {
    const int64_t n = 2 * static_cast<int64_t>(a.D);
    norm_sum_kernel<<<static_cast<unsigned>((n + kSumCols - 1) / kSumCols), kSumCols * kSumGroups, 0, stream>>>(
        part, nparts, a.D, a.dweight, a.dbias);
  }
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  if (a.x_bf16)
    a.y_bf16 ? norm_call<bf16, bf16>(a, stream) : norm_call<bf16, float>(a, stream);
  else
    a.y_bf16 ? norm_call<float, bf16>(a, stream) : norm_call<float, float>(a, stream);
  return hipGetLastError();
}

size_t norm_grad_workspace_bytes(int64_t T, int D) {
  // one partial row pair per workgroup; the most that any plan makes
  const int64_t blocks = T < kGradBlocks ? T : kGradBlocks;
  Carver c{nullptr};
  c.take<float>(static_cast<size_t>(blocks) * 2 * D);
  return c.size();
}

hipError_t launch_norm_grad(const NormGradArgs& a, hipStream_t stream) {
  if (a.x_bf16)
    a.dy_bf16 ? norm_grad_call<bf16, bf16>(a, stream) : norm_grad_call<bf16, float>(a, stream);
  else
    a.dy_bf16 ? norm_grad_call<float, bf16>(a, stream) : norm_grad_call<float, float>(a, stream);
  return hipGetLastError();
}

}  // namespace emb
