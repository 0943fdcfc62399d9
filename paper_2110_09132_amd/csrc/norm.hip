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

// The forward pass.  Every workgroup takes the next rows in memory and ends:
// the memory then sees one front of accesses that moves through it, which it
// serves faster than the many fronts of workgroups that stride over the rows
// (plain copies of 256 MB each way, 16 bytes per lane, streaming: 6.5 TB/s, and
// 5.7 to 6.3 with 1024 to 8192 workgroups that stride).  kR rows
// are in flight at once, and share the reads of the weight and the bias (from
// the L2: 8 D bytes, as much as or more than a row itself).  Measured (8192 x
// 8192 bf16): one row 62 us, two 50 us (5.4 TB/s, as torch's copies reach),
// four 54 us; 32768 x 2048: 51, 49, 51.  Looked-up rows are taken one at a time
// (16384 rows of 1024 fp32, to bf16: one 13.6 us, two 13.9 us), as are few
// rows, which have to spread over the chip.  y goes out with streaming stores
// (two to five percent), x comes in with streaming loads unless it is looked
// up: a batch's frequent rows are worth keeping (13.6 against 18.6 us).
constexpr int kThreads = 256;
constexpr int64_t kManyBlocks = 1024;
template <typename XT, typename YT, int kE, int kL, int kNV, int kW, int kR>
__global__ __launch_bounds__(kW > 1 ? kW * kWave : kThreads) void norm_kernel(
    Source<XT> src, int64_t begin, int64_t T, int D, const float* __restrict__ weight, const float* __restrict__ bias,
    float eps, Rows<YT> y, float* __restrict__ mean_out, float* __restrict__ rstd_out, int32_t* status) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kRows = kW > 1 ? 1 : kThreads / kLanes;
  __shared__ float red[2][kW > 1 ? kW : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  const int sub = static_cast<int>(threadIdx.x) / kLanes;
  const float fD = static_cast<float>(D);
  const Columns<kE, kLanes, kNV> cols{lane, D};
  bool bad = false;
  const int64_t t0 = begin + (static_cast<int64_t>(blockIdx.x) * kRows + sub) * kR;
  Vec<XT, kE> x[kR][kNV];
#pragma unroll
  for (int r = 0; r < kR; ++r) {  // rows past the last read the last
    bool none = false;
    const XT* row = src.row(min(t0 + r, T - 1), none);
    if (none) row = src.p;
    // (the statements that keep the branches apart: the compiler would make one
    // access of the two, which differ in their cache policy only)
    if (src.ids == nullptr) {
      asm volatile("");
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template load<true>(row, k, x[r][k]);
      asm volatile("");
    } else {
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template load<false>(row, k, x[r][k]);
    }
    if (none) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) x[r][k].clear();
    }
    bad |= none;
  }
  float w[kNV][kE], b[kNV][kE];
#pragma unroll
  for (int k = 0; k < kNV; ++k) {
    cols.load(weight, k, 1.0f, w[k]);
    cols.load(bias, k, 0.0f, b[k]);
  }
#pragma unroll
  for (int r = 0; r < kR; ++r) {
    const int64_t t = t0 + r;
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k)
#pragma unroll
      for (int e = 0; e < kE; ++e) s += cols.own(k, e) ? x[r][k][e] : 0.0f;
    const float mean = row_sum<kL, kW>(s, red, 0) / fD;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k)
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float d = cols.own(k, e) ? x[r][k][e] - mean : 0.0f;
        s += d * d;
      }
    const float rstd = 1.0f / sqrtf(row_sum<kL, kW>(s, red, 1) / fD + eps);
    if (t < T) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        float v[kE];
#pragma unroll
        for (int e = 0; e < kE; ++e) v[e] = (x[r][k][e] - mean) * rstd * w[k][e] + b[k][e];
        cols.template store<true>(y.p + t * y.ld, k, v);
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
// A lane has up to kGradElems elements of a row, in two buffers; rows of more
// than 8 waves' worth take more elements in one buffer (two would not fit the
// registers).  Measured (65536 x 1024 bf16, 403 MB): 135 us with one buffer and
// half the waves, 72 us so (5.6 TB/s; torch's copies reach 5.4); 32768 x
// 2048: 92 us with 32 elements per lane in one buffer, 71 us so.
constexpr int kGradThreads = 512;
constexpr int kGradElems = 16;
template <typename XT, typename GT, int kE, int kL, int kNV, int kW>
__global__ __launch_bounds__(kGradThreads) void norm_grad_kernel(
    Rows<const GT> dy, Source<XT> src, int64_t T, int D, const float* __restrict__ weight,
    const float* __restrict__ mean_in, const float* __restrict__ rstd_in, Rows<GT> dx, float* __restrict__ part,
    int32_t* status) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kRows = kGradThreads / kLanes;
  constexpr int kWaves = kGradThreads / kWave;
  constexpr int kJoin = kWaves / kW;  // groups of kW waves that hold sums of the same columns
  __shared__ float2 red[2][kWaves];
  __shared__ float join[kJoin > 1 ? kJoin : 1][kJoin > 1 ? kLanes * kNV * kE : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes;
  const int sub = static_cast<int>(threadIdx.x) / kLanes;
  const float fD = static_cast<float>(D);
  const Columns<kE, kLanes, kNV> cols{lane, D};
  bool bad = false;
  float dw[kNV][kE] = {}, db[kNV][kE] = {}, w[kNV][kE];
  int slot = 0;
  constexpr bool kAhead = kNV * kE <= kGradElems;
  // two rows in registers: the loads of the next row are in flight while the current one is worked on
  struct Buf {
    Vec<XT, kE> x[kNV];
    Vec<GT, kE> g[kNV];
    float mean, rstd;
  } A, B;
  const int64_t step = static_cast<int64_t>(gridDim.x) * kRows;
  int64_t id_next = 0;  // table row of the row after the next load, read one load ahead
  const auto read_id = [&](int64_t t) { id_next = src.ids != nullptr && t < T ? src.ids[t] : t; };
  const auto load = [&](int64_t t, Buf& u) {  // rows past the last read a valid row, and count as zeros
    const bool live = t < T;
    const int64_t id = id_next;
    const bool found = src.ids == nullptr || (id >= 0 && id < src.V);
    bad |= live && !found;
    const XT* row = src.p + (live && found ? id : 0) * src.ld;
    const GT* grow = dy.p + (live ? t : 0) * dy.ld;
    read_id(t + step);
    u.mean = live ? mean_in[t] : 0.0f;
    u.rstd = live ? rstd_in[t] : 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) cols.template load<false>(row, k, u.x[k]);
#pragma unroll
    for (int k = 0; k < kNV; ++k) cols.template load<true>(grow, k, u.g[k]);
    if (!live || !found) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        u.x[k].clear();
        if (!live) u.g[k].clear();
      }
    }
  };
  const auto work = [&](int64_t t, Buf& u) {
    float xh[kNV][kE], g[kNV][kE];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        xh[k][e] = (u.x[k][e] - u.mean) * u.rstd;
        g[k][e] = u.g[k][e];
        dw[k][e] += g[k][e] * xh[k][e];
        db[k][e] += g[k][e];
        g[k][e] *= w[k][e];
        s1 += cols.own(k, e) ? g[k][e] : 0.0f;
        s2 += cols.own(k, e) ? g[k][e] * xh[k][e] : 0.0f;
      }
    }
    row_sum2<kL, kW, kWaves>(s1, s2, red, slot);
    slot ^= 1;
    const float c1 = s1 / fD, c2 = s2 / fD;
    if (t < T && dx.p != nullptr) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
#pragma unroll
        for (int e = 0; e < kE; ++e) g[k][e] = u.rstd * (g[k][e] - c1 - xh[k][e] * c2);
        cols.template store<true>(dx.p + t * dx.ld, k, g[k]);
      }
    }
  };
  int64_t t0 = static_cast<int64_t>(blockIdx.x) * kRows;  // first row of the workgroup's group: the same in all lanes
  read_id(t0 + sub);
  load(t0 + sub, A);
#pragma unroll
  for (int k = 0; k < kNV; ++k) cols.load(weight, k, 1.0f, w[k]);
  while (true) {
    if (kAhead) load(t0 + step + sub, B);
    work(t0 + sub, A);
    t0 += step;
    if (t0 >= T) break;
    load(t0 + (kAhead ? step : 0) + sub, A);
    if (kAhead) {
      work(t0 + sub, B);
      t0 += step;
      if (t0 >= T) break;
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
    if constexpr (kJoin > 1) {  // the rows of the workgroup
      const int g = static_cast<int>(threadIdx.x) / (kWave * kW);
      if (static_cast<int>(threadIdx.x) % (kWave * kW) < kLanes) {
#pragma unroll
        for (int k = 0; k < kNV; ++k)
#pragma unroll
          for (int e = 0; e < kE; ++e) join[g][cols.first(k) + e] = a[k][e];
      }
      __syncthreads();
      for (int c = static_cast<int>(threadIdx.x); c < D; c += kGradThreads) {
        float s = join[0][c];
#pragma unroll
        for (int i = 1; i < kJoin; ++i) s += join[i][c];
        out[static_cast<size_t>(which) * D + c] = s;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template store<false>(out + static_cast<size_t>(which) * D, k, a[k]);
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
  __shared__ float2 red[2][kLoopWaves];
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
    row_sum2<kWave, kLoopWaves, kLoopWaves>(s1, s2, red, slot);
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
// The launch's first workgroup is number `first` of all.
constexpr int kSumCols = 32;
constexpr int kSumGroups = 32;
__global__ __launch_bounds__(kSumCols* kSumGroups) void norm_sum_kernel(const float* __restrict__ part, int nparts,
                                                                        int D, int first, float* __restrict__ dw,
                                                                        float* __restrict__ db) {
  __shared__ float red[kSumGroups][kSumCols + 1];
  const int col = static_cast<int>(threadIdx.x) % kSumCols, g = static_cast<int>(threadIdx.x) / kSumCols;
  const int64_t c0 = (static_cast<int64_t>(first) + blockIdx.x) * kSumCols, c = c0 + col;
  const int64_t n = 2 * static_cast<int64_t>(D);
  float s = 0.0f;
  if (c < n) {
#pragma unroll 16
    for (int p = g; p < nparts; p += kSumGroups) s += part[p * n + c];
  }
  red[g][col] = s;
  __syncthreads();
  // thread (col, g) now takes group `col` of column `g`: a column's groups are neighbouring lanes
  static_assert(kSumCols == kSumGroups, "a square of threads");
  s = group_sum<kSumGroups>(red[col][g]);
  const int64_t o = c0 + g;
  if (col == 0 && o < n) {
    float* out = o < D ? dw : db;
    if (out != nullptr) out[o < D ? o : o - D] = s;
  }
}

// Workgroups of the backward pass, and so the number of partial rows: two per
// CU; one where a row has 1024 elements or more, whose partial rows cost more
// than the second workgroup brings (8192 x 8192 bf16: 85 us with 512, 77 us with
// 256 workgroups, sums included; 60000 x 256 fp32: 34 and 37 us).  No more than
// two fit a CU's registers (768: 40 us, 1024: 37 us).
constexpr int kGradBlocks = 512;
int grad_blocks(int64_t T, int D, int rows_per_block) {
  const int64_t b = (T + rows_per_block - 1) / rows_per_block;
  const int64_t most = D >= 1024 ? kGradBlocks / 2 : kGradBlocks;
  return static_cast<int>(b < most ? b : most);
}
int rows_per_block(const RowPlan& pl, int threads) { return threads / (pl.waves * pl.lanes); }

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

template <typename XT, typename YT, int kE>
void norm_call(const NormArgs& a, hipStream_t stream) {
  const Source<XT> src{static_cast<const XT*>(a.x), a.ldx, a.ids, a.V};
  const Rows<YT> y{static_cast<YT*>(a.y), a.ldy};
  const RowPlan pl = plan_row(a.D, kE, kMaxElems);
  const float eps = static_cast<float>(a.eps);
  if (pl.waves == 0) {
    norm_loop_kernel<XT, YT><<<grid_for(a.T, kMaxBlocks), kLoopWaves * kWave, 0, stream>>>(
        src, a.T, a.D, a.weight, a.bias, eps, y, a.mean, a.rstd, a.status);
    return;
  }
  const int64_t each = pl.waves > 1 ? 1 : rows_per_block(pl, kThreads);
  const bool two = a.ids == nullptr && a.T > 2 * each * (kManyBlocks - 1);
  const int64_t rows = two ? 2 * each : each;  // per workgroup
  with_shape<kE, kMaxElems>(pl, [&](auto L, auto NV, auto W) {
    const auto kernel = two ? norm_kernel<XT, YT, kE, L.value, NV.value, W.value, 2>
                            : norm_kernel<XT, YT, kE, L.value, NV.value, W.value, 1>;
    for (int64_t begin = 0; begin < a.T; begin += rows * kMaxBlocks)
      kernel<<<grid_for((a.T - begin + rows - 1) / rows, kMaxBlocks), W.value > 1 ? W.value * kWave : kThreads, 0,
               stream>>>(src, begin, a.T, a.D, a.weight, a.bias, eps, y, a.mean, a.rstd, a.status);
  });
}

template <typename XT, typename GT, int kE>
void norm_grad_call(const NormGradArgs& a, hipStream_t stream) {
  const Source<XT> src{static_cast<const XT*>(a.x), a.ldx, a.ids, a.V};
  const Rows<const GT> dy{static_cast<const GT*>(a.dy), a.lddy};
  const Rows<GT> dx{static_cast<GT*>(a.dx), a.lddx};
  const bool params = a.dweight != nullptr || a.dbias != nullptr;
  float* part = params ? static_cast<float*>(a.workspace) : nullptr;
  const RowPlan pl = plan_row(a.D, kE, kGradElems);
  int nparts = 0;
  if (a.T > 0 && pl.waves == 0) {
    if (params) {  // first: dx may be written over dy
      nparts = grad_blocks(a.T, a.D, 16);
      norm_columns_kernel<XT, GT><<<dim3((a.D + 4 * kThreads - 1) / (4 * kThreads), nparts), kThreads, 0, stream>>>(
          dy, src, a.T, a.D, a.mean, a.rstd, part, a.status);
    }
    if (a.dx != nullptr)
      norm_grad_loop_kernel<XT, GT><<<grid_for(a.T, kMaxBlocks), kLoopWaves * kWave, 0, stream>>>(
          dy, src, a.T, a.D, a.weight, a.mean, a.rstd, dx, a.status);
  } else if (a.T > 0) {
    nparts = grad_blocks(a.T, a.D, rows_per_block(pl, kGradThreads));
    with_shape<kE, kGradElems>(pl, [&](auto L, auto NV, auto W) {
      norm_grad_kernel<XT, GT, kE, L.value, NV.value, W.value>
          <<<nparts, kGradThreads, 0, stream>>>(dy, src, a.T, a.D, a.weight, a.mean, a.rstd, dx, part, a.status);
    });
  }
  if (params) {
    // a launch holds less than 2^32 threads
    const int64_t blocks = (2 * static_cast<int64_t>(a.D) + kSumCols - 1) / kSumCols;
    for (int64_t first = 0; first < blocks; first += kMaxBlocks)
      norm_sum_kernel<<<grid_for(blocks - first, kMaxBlocks), kSumCols * kSumGroups, 0, stream>>>(
          part, nparts, a.D, static_cast<int>(first), a.dweight, a.dbias);
  }
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  if (a.x_bf16 && a.y_bf16)
    norm_call<bf16, bf16, 8>(a, stream);
  else if (a.x_bf16)
    norm_call<bf16, float, 4>(a, stream);
  else
    a.y_bf16 ? norm_call<float, bf16, 4>(a, stream) : norm_call<float, float, 4>(a, stream);
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
  if (a.x_bf16 && a.dy_bf16)
    norm_grad_call<bf16, bf16, 8>(a, stream);
  else if (a.x_bf16)
    norm_grad_call<bf16, float, 4>(a, stream);
  else
    a.dy_bf16 ? norm_grad_call<float, bf16, 4>(a, stream) : norm_grad_call<float, float, 4>(a, stream);
  return hipGetLastError();
}

}  // namespace emb
