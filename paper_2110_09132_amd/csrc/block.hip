// The norms before and after a block, with its dropout, gate and residual scale.
//
//   n = N_post(branch);  h = alpha x + gate keep n s;  y = N_pre(h)          s = 1 / (1 - q)
//   d = dh + N_pre'(dy);  dx = alpha d
//   dn = gate keep d s;   dbranch = N_post'(dn);  dgate = sum keep d n s
//   N'(g) = rstd (g w - sum g w / D - xh sum (g w xh) / D),  dw = sum g xh,  db = sum g
//
// Bound by memory: forward, x and branch are read and h and y written once;
// backward, dh, dy, h and branch are read, dx and dbranch written.  n, the mask
// and the normalised rows are formed again instead of being kept.
#include "dropout.h"
#include "rows.h"

namespace emb {
namespace {

// Sum of two values over the workgroup, in every lane; `slot` alternates so that one barrier is enough.
constexpr int kWaves = 16;
constexpr int kWide = kWaves * kWave;
struct Sums {
  float2 (*red)[kWaves];
  int slot;
  __device__ __forceinline__ void operator()(float& a, float& b) {
    a = group_sum<kWave>(a);
    b = group_sum<kWave>(b);
    if (lane_id() == 0) red[slot][threadIdx.x / kWave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      a += red[slot][w].x;
      b += red[slot][w].y;
    }
    slot ^= 1;
  }
};

__device__ __forceinline__ int64_t gate_row(int64_t t, int64_t gate_rows) {
  return gate_rows > 0 ? static_cast<uint32_t>(t) / static_cast<uint32_t>(gate_rows) : 0;
}

// A row's part of four elements from column c on.
__device__ __forceinline__ void param4(const float* p, int c, int D, float fill, float (&v)[4]) {
  load_part(p + c, p != nullptr ? D - c : 0, fill, v);
}

// Whether a row is written over itself and has a vector that Columns moves back, which then reads what another wave may
// write: all of the row's waves have to have read it first.  The sums of a norm see to that; without one it takes a
// barrier, which costs the rows of the backward pass their overlap (16384 x 8192 bf16, no norms: 182 us, with a barrier
// in every row 202).
template <int kE>
__device__ __forceinline__ bool over_itself(const void* in, const void* out, int D) {
  return in == out && D % kE != 0;
}

// ---------------------------------------------------------------- rows that fit registers
// Forward.  A workgroup takes the next rows in memory and ends; a row and its
// branch stay in registers, h replaces them.
constexpr int kThreads = 256;
template <typename ST, typename BT, int kE, int kL, int kNV, int kW>
__global__ __launch_bounds__(kW > 1 ? kW * kWave : kThreads) void block_kernel(const emb_block_norm_args a,
                                                                               DropMask mask, int64_t begin) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kRows = kW > 1 ? 1 : kThreads / kLanes;
  __shared__ float red[2][kW > 1 ? kW : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes, sub = static_cast<int>(threadIdx.x) / kLanes;
  const int D = a.D;
  const float fD = static_cast<float>(D), eps = static_cast<float>(a.eps), alpha = static_cast<float>(a.alpha);
  const Columns<kE, kLanes, kNV> cols{lane, D};
  const int64_t row = begin + static_cast<int64_t>(blockIdx.x) * kRows + sub;
  const bool live = row < a.T;
  const int64_t t = live ? row : a.T - 1;
  Vec<ST, kE> x[kNV];
  Vec<BT, kE> br[kNV];
#pragma unroll
  for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const BT*>(a.branch) + t * a.ldb, k, br[k]);
#pragma unroll
  for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const ST*>(a.x) + t * a.ldx, k, x[k]);
  const float* gate = a.gate != nullptr ? a.gate + gate_row(t, a.gate_rows) * D : nullptr;
  const auto statistics = [&](auto&& at, float& mean, float& rstd, float* out) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k)
#pragma unroll
      for (int e = 0; e < kE; ++e) s += cols.own(k, e) ? at(k, e) : 0.0f;
    mean = row_sum<kL, kW>(s, red, 0) / fD;
    s = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k)
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        const float d = cols.own(k, e) ? at(k, e) - mean : 0.0f;
        s += d * d;
      }
    rstd = 1.0f / sqrtf(row_sum<kL, kW>(s, red, 1) / fD + eps);
    if (live && lane == 0) {
      out[t] = mean;
      out[a.T + t] = rstd;
    }
  };
  float mean = 0.0f, rstd = 1.0f;
  if (a.post_stats != nullptr)
    statistics([&](int k, int e) { return br[k][e]; }, mean, rstd, a.post_stats);
  else if (kW > 1 && over_itself<kE>(a.x, a.h, D))
    __syncthreads();
  const uint64_t key = mask.cut != 0 ? mask_key(mask) : 0;
  const int64_t per = (static_cast<int64_t>(D) + 3) / 4;
  float h[kNV][kE];
#pragma unroll
  for (int k = 0; k < kNV; ++k) {
    float n[kE], w[kE], b[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) n[e] = br[k][e];
    if (a.post_stats != nullptr) {
      cols.load(a.post_weight, k, 1.0f, w);
      cols.load(a.post_bias, k, 0.0f, b);
#pragma unroll
      for (int e = 0; e < kE; ++e) n[e] = (n[e] - mean) * rstd * w[e] + b[e];
    }
    if (mask.cut != 0) apply_mask(mask, key, t, per, cols.first(k), n);
    cols.load(gate, k, 1.0f, w);
#pragma unroll
    for (int e = 0; e < kE; ++e) h[k][e] = alpha * x[k][e] + w[e] * n[e];
    if (live) cols.template store<true>(static_cast<ST*>(a.h) + t * a.ldh, k, h[k]);
  }
  if (a.pre_stats == nullptr) return;
  statistics([&](int k, int e) { return h[k][e]; }, mean, rstd, a.pre_stats);
  if (!live) return;
#pragma unroll
  for (int k = 0; k < kNV; ++k) {
    float w[kE], b[kE];
    cols.load(a.pre_weight, k, 1.0f, w);
    cols.load(a.pre_bias, k, 0.0f, b);
#pragma unroll
    for (int e = 0; e < kE; ++e) h[k][e] = (h[k][e] - mean) * rstd * w[e] + b[e];
    cols.template store<true>(static_cast<BT*>(a.y) + t * a.ldy, k, h[k]);
  }
}

// Backward.  A workgroup holds the column sums of its rows in registers; at the
// end the rows that share a workgroup are joined into one partial row of part [gridDim.x][5][D] (dpre_weight,
// dpre_bias, dpost_weight, dpost_bias, dgate), which block_sum_kernel adds up in
// workgroup order.  kGroups: groups of gate_rows rows have gates of their own.
// Every place for a row in a workgroup then takes `run` rows after another, and
// writes its sum for dgate where a group ends: to dgate itself where the whole
// group is its own, else to one of its two rows of pieces [place][2][D] (0: the
// group that its first row is in, 1: the one that its last row is in).
constexpr int grad_threads(int waves) { return waves > 4 ? 512 : 256; }
constexpr int kGradMost = 16;  // elements of a lane
constexpr int kGradFew = 8;    // up to this many, three workgroups of 256 threads have their registers on a CU, else two
template <typename ST, typename BT, int kE, int kL, int kNV, int kW, bool kGroups>
__global__ __launch_bounds__(grad_threads(kW), kNV* kE <= kGradFew ? 3 : 2) void block_grad_kernel(
    const emb_block_norm_grad_args a, DropMask mask, int64_t run, float* __restrict__ part, float* __restrict__ pieces) {
  constexpr int kLanes = kW > 1 ? kW * kWave : kL;
  constexpr int kThreadsHere = grad_threads(kW);
  constexpr int kRows = kThreadsHere / kLanes;
  constexpr int kGradWaves = kThreadsHere / kWave;
  constexpr int kJoin = kGradWaves / kW;  // groups of kW waves that hold sums of the same columns
  __shared__ float2 red[2][kGradWaves];
  __shared__ float join[kJoin > 1 ? kJoin : 1][kJoin > 1 ? kLanes * kNV * kE : 1];
  const int lane = static_cast<int>(threadIdx.x) % kLanes, sub = static_cast<int>(threadIdx.x) / kLanes;
  const int D = a.D;
  const float fD = static_cast<float>(D), alpha = static_cast<float>(a.alpha);
  const Columns<kE, kLanes, kNV> cols{lane, D};
  const bool pre = a.pre_stats != nullptr, post = a.post_stats != nullptr;
  const uint64_t key = mask_key(mask);
  const int64_t per = (static_cast<int64_t>(D) + 3) / 4;
  const int64_t place = static_cast<int64_t>(blockIdx.x) * kRows + sub;
  const int64_t begin = kGroups ? place * run : place;
  const int64_t end = kGroups ? min(static_cast<int64_t>(a.T), begin + run) : a.T;
  const int64_t step = kGroups ? 1 : static_cast<int64_t>(gridDim.x) * kRows;
  float sums[5][kNV][kE] = {};
  int slot = 0;
  struct Buf {
    Vec<ST, kE> dh[kNV], h[kNV];
    Vec<BT, kE> dy[kNV], b[kNV];
    float hmean, hrstd, bmean, brstd;
  };
  const auto load = [&](int64_t row, Buf& u) {  // rows past the last read a valid row, and count as zeros
    const bool live = row < end;
    const int64_t t = live ? row : 0;
    u.hmean = pre && live ? a.pre_stats[t] : 0.0f;
    u.hrstd = pre && live ? a.pre_stats[a.T + t] : 0.0f;
    u.bmean = post && live ? a.post_stats[t] : 0.0f;
    u.brstd = post && live ? a.post_stats[a.T + t] : 0.0f;
    if (pre) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const BT*>(a.dy) + t * a.lddy, k, u.dy[k]);
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const ST*>(a.h) + t * a.ldh, k, u.h[k]);
    }
    if (a.dh != nullptr) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const ST*>(a.dh) + t * a.lddh, k, u.dh[k]);
    }
#pragma unroll
    for (int k = 0; k < kNV; ++k) cols.template load<true>(static_cast<const BT*>(a.branch) + t * a.ldb, k, u.b[k]);
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      if (!live || !pre) {
        u.dy[k].clear();
        u.h[k].clear();
      }
      if (!live || a.dh == nullptr) u.dh[k].clear();
      if (!live) u.b[k].clear();
    }
  };
  const auto work = [&](int64_t t, Buf& u, const uint64_t(&state)[kNV]) {
    const bool live = t < end;
    float d[kNV][kE], xh[kNV][kE], w[kE], v[kE];
    float c1 = 0.0f, c2 = 0.0f;
    if (pre) {
#pragma unroll
      for (int k = 0; k < kNV; ++k) {
        cols.load(a.pre_weight, k, 1.0f, w);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          xh[k][e] = (u.h[k][e] - u.hmean) * u.hrstd;
          const float dy = u.dy[k][e], g = dy * w[e];
          sums[0][k][e] += dy * xh[k][e];
          sums[1][k][e] += dy;
          d[k][e] = g;
          c1 += cols.own(k, e) ? g : 0.0f;
          c2 += cols.own(k, e) ? g * xh[k][e] : 0.0f;
        }
      }
      row_sum2<kL, kW, kGradWaves>(c1, c2, red, slot);
      slot ^= 1;
      c1 /= fD;
      c2 /= fD;
    } else if (kW > 1 && over_itself<kE>(a.dh, a.dx, D)) {
      __syncthreads();
    }
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        d[k][e] = pre ? u.dh[k][e] + u.hrstd * (d[k][e] - c1 - xh[k][e] * c2) : u.dh[k][e];
        v[e] = alpha * d[k][e];
      }
      if (live && a.dx != nullptr) cols.template store<true>(static_cast<ST*>(a.dx) + t * a.lddx, k, v);
    }
    const float* gate = a.gate != nullptr ? a.gate + gate_row(live ? t : 0, a.gate_rows) * D : nullptr;
    float(&bh)[kNV][kE] = xh;
    float c3 = 0.0f, c4 = 0.0f;
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      float gt[kE];
      bool keep[kE];
      if (mask.cut != 0) {
        mask_bits(mask.cut, state[k], cols.first(k) % 4, keep);
      } else {
#pragma unroll
        for (int e = 0; e < kE; ++e) keep[e] = true;
      }
      cols.load(gate, k, 1.0f, gt);
      if (post) {
        cols.load(a.post_weight, k, 1.0f, w);
        cols.load(a.post_bias, k, 0.0f, v);
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const float ds = keep[e] ? d[k][e] * mask.scale : 0.0f, dn = ds * gt[e], g = dn * w[e];
          bh[k][e] = (u.b[k][e] - u.bmean) * u.brstd;
          sums[2][k][e] += dn * bh[k][e];
          sums[3][k][e] += dn;
          sums[4][k][e] += ds * (bh[k][e] * w[e] + v[e]);
          c3 += cols.own(k, e) ? g : 0.0f;
          c4 += cols.own(k, e) ? g * bh[k][e] : 0.0f;
          d[k][e] = g;
        }
      } else {  // what is dropped is not used, whatever it is
#pragma unroll
        for (int e = 0; e < kE; ++e) {
          const float ds = keep[e] ? d[k][e] * mask.scale : 0.0f;
          sums[4][k][e] += keep[e] ? ds * u.b[k][e] : 0.0f;
          d[k][e] = ds * gt[e];
        }
      }
    }
    if (post) {
      row_sum2<kL, kW, kGradWaves>(c3, c4, red, slot);
      slot ^= 1;
      c3 /= fD;
      c4 /= fD;
    }
#pragma unroll
    for (int k = 0; k < kNV; ++k) {
      if (post) {
#pragma unroll
        for (int e = 0; e < kE; ++e) d[k][e] = u.brstd * (d[k][e] - c3 - bh[k][e] * c4);
      }
      if (live && a.dbranch != nullptr) cols.template store<true>(static_cast<BT*>(a.dbranch) + t * a.lddb, k, d[k]);
    }
    if constexpr (kGroups) {
      const uint32_t rows = static_cast<uint32_t>(a.gate_rows), row = static_cast<uint32_t>(t), g = row / rows;
      if (live && (t + 1 == end || (row + 1) / rows != g)) {
        const bool whole = static_cast<int64_t>(g) * rows >= begin &&
                           min(static_cast<int64_t>(a.T), (static_cast<int64_t>(g) + 1) * rows) <= end;
        const int which = g == static_cast<uint32_t>(begin) / rows ? 0 : 1;
        float* out = whole ? a.dgate + static_cast<int64_t>(g) * D : pieces + (place * 2 + which) * D;
#pragma unroll
        for (int k = 0; k < kNV; ++k) {
          cols.template store<false>(out, k, sums[4][k]);
#pragma unroll
          for (int e = 0; e < kE; ++e) sums[4][k][e] = 0.0f;
        }
      }
    }
  };
  // the same number of rounds in every place: the row sums need all waves
  const int64_t rounds = kGroups ? run : (a.T - static_cast<int64_t>(blockIdx.x) * kRows + step - 1) / step;
  uint64_t state[kNV];
#pragma unroll
  for (int k = 0; k < kNV; ++k) state[k] = mask_state(key, begin * per + cols.first(k) / 4);
  Buf u;
  for (int64_t i = 0, t = begin; i < rounds; ++i, t += step) {
    load(t, u);
    work(t, u, state);
#pragma unroll
    for (int k = 0; k < kNV; ++k) state[k] += static_cast<uint64_t>(step * per) * kGamma;
  }
  if (part == nullptr) return;
  float* out = part + static_cast<size_t>(blockIdx.x) * 5 * D;
#pragma unroll
  for (int which = 0; which < (kGroups ? 4 : 5); ++which) {
    float(&s)[kNV][kE] = sums[which];
    if constexpr (kL < kWave) {  // the rows of a wave
#pragma unroll
      for (int k = 0; k < kNV; ++k)
#pragma unroll
        for (int e = 0; e < kE; ++e)
          for (int m = kL; m < kWave; m *= 2) s[k][e] += __shfl_xor(s[k][e], m, kWave);
    }
    if constexpr (kJoin > 1) {  // the rows of the workgroup
      const int g = static_cast<int>(threadIdx.x) / (kWave * kW);
      if (static_cast<int>(threadIdx.x) % (kWave * kW) < kLanes) {
#pragma unroll
        for (int k = 0; k < kNV; ++k)
#pragma unroll
          for (int e = 0; e < kE; ++e)
            if (cols.first(k) + e < D) join[g][cols.first(k) + e] = s[k][e];
      }
      __syncthreads();
      for (int c = static_cast<int>(threadIdx.x); c < D; c += kThreadsHere) {
        float v = join[0][c];
#pragma unroll
        for (int i = 1; i < kJoin; ++i) v += join[i][c];
        out[static_cast<size_t>(which) * D + c] = v;
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int k = 0; k < kNV; ++k) cols.template store<false>(out + static_cast<size_t>(which) * D, k, s[k]);
    }
  }
}

// ---------------------------------------------------------------- rows of any width
// One workgroup per row, which reads the row again for every pass over it.
template <typename ST, typename BT>
__global__ __launch_bounds__(kWide) void block_loop_kernel(const emb_block_norm_args a, DropMask mask) {
  __shared__ float2 red[2][kWaves];
  Sums sums{red, 0};
  const int D = a.D, step = kWide * 4, c_first = static_cast<int>(threadIdx.x) * 4;
  const float fD = static_cast<float>(D), eps = static_cast<float>(a.eps), alpha = static_cast<float>(a.alpha);
  const uint64_t key = mask_key(mask);
  const int64_t per = (static_cast<int64_t>(D) + 3) / 4;
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    const ST* x = static_cast<const ST*>(a.x) + t * a.ldx;
    const BT* br = static_cast<const BT*>(a.branch) + t * a.ldb;
    const float* gate = a.gate != nullptr ? a.gate + gate_row(t, a.gate_rows) * D : nullptr;
    float mean = 0.0f, rstd = 1.0f, none = 0.0f;
    if (a.post_stats != nullptr) {
      float s = 0.0f, v[4];
      for (int c = c_first; c < D; c += step) {
        load_part(br + c, D - c, 0.0f, v);
        s += (v[0] + v[1]) + (v[2] + v[3]);
      }
      sums(s, none);
      mean = s / fD;
      s = 0.0f;
      for (int c = c_first; c < D; c += step) {
        load_part(br + c, D - c, 0.0f, v);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float d = c + e < D ? v[e] - mean : 0.0f;
          s += d * d;
        }
      }
      sums(s, none);
      rstd = 1.0f / sqrtf(s / fD + eps);
      if (threadIdx.x == 0) {
        a.post_stats[t] = mean;
        a.post_stats[a.T + t] = rstd;
      }
    }
    const auto row = [&](int c, float(&h)[4]) {  // h from column c on
      float n[4], w[4], b[4];
      load_part(x + c, D - c, 0.0f, h);
      load_part(br + c, D - c, 0.0f, n);
      if (a.post_stats != nullptr) {
        param4(a.post_weight, c, D, 1.0f, w);
        param4(a.post_bias, c, D, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) n[e] = (n[e] - mean) * rstd * w[e] + b[e];
      }
      if (mask.cut != 0) apply_mask(mask, key, t, per, c, n);
      param4(gate, c, D, 1.0f, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = alpha * h[e] + w[e] * n[e];
    };
    float hmean = 0.0f, hrstd = 1.0f, h[4];
    if (a.pre_stats != nullptr) {
      float s = 0.0f;
      for (int c = c_first; c < D; c += step) {
        row(c, h);
#pragma unroll
        for (int e = 0; e < 4; ++e) s += c + e < D ? h[e] : 0.0f;
      }
      sums(s, none);
      hmean = s / fD;
      s = 0.0f;
      for (int c = c_first; c < D; c += step) {
        row(c, h);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float d = c + e < D ? h[e] - hmean : 0.0f;
          s += d * d;
        }
      }
      sums(s, none);
      hrstd = 1.0f / sqrtf(s / fD + eps);
      if (threadIdx.x == 0) {
        a.pre_stats[t] = hmean;
        a.pre_stats[a.T + t] = hrstd;
      }
    }
    for (int c = c_first; c < D; c += step) {  // h may be x and y branch: a lane writes only what it has read
      row(c, h);
      store_part(static_cast<ST*>(a.h) + t * a.ldh + c, D - c, h);
      if (a.pre_stats != nullptr) {
        float w[4], b[4];
        param4(a.pre_weight, c, D, 1.0f, w);
        param4(a.pre_bias, c, D, 0.0f, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = (h[e] - hmean) * hrstd * w[e] + b[e];
        store_part(static_cast<BT*>(a.y) + t * a.ldy + c, D - c, h);
      }
    }
  }
}

// What the backward pass forms of a row again, from column c on.
template <typename ST, typename BT>
struct GradRow {
  const emb_block_norm_grad_args& a;
  const DropMask& mask;
  uint64_t key;
  int64_t t, per;
  float c1, c2;  // sums of N_pre', once they are known
  float hmean, hrstd, bmean, brstd;
  __device__ GradRow(const emb_block_norm_grad_args& args, const DropMask& m, uint64_t k, int64_t row)
      : a(args), mask(m), key(k), t(row), per((static_cast<int64_t>(args.D) + 3) / 4), c1(0.0f), c2(0.0f) {
    hmean = a.pre_stats != nullptr ? a.pre_stats[t] : 0.0f;
    hrstd = a.pre_stats != nullptr ? a.pre_stats[a.T + t] : 1.0f;
    bmean = a.post_stats != nullptr ? a.post_stats[t] : 0.0f;
    brstd = a.post_stats != nullptr ? a.post_stats[a.T + t] : 1.0f;
  }
  // dy, and h normalised
  __device__ __forceinline__ void pre(int c, float (&dy)[4], float (&xh)[4]) const {
    load_part(static_cast<const BT*>(a.dy) + t * a.lddy + c, a.D - c, 0.0f, dy);
    load_part(static_cast<const ST*>(a.h) + t * a.ldh + c, a.D - c, hmean, xh);
#pragma unroll
    for (int e = 0; e < 4; ++e) xh[e] = (xh[e] - hmean) * hrstd;
  }
  // the gradient of h
  __device__ __forceinline__ void d(int c, float (&out)[4]) const {
    load_part(static_cast<const ST*>(a.dh) + t * a.lddh + c, a.dh != nullptr ? a.D - c : 0, 0.0f, out);
    if (a.pre_stats == nullptr) return;
    float dy[4], xh[4], w[4];
    pre(c, dy, xh);
    param4(a.pre_weight, c, a.D, 1.0f, w);
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] += hrstd * (dy[e] * w[e] - c1 - xh[e] * c2);
  }
  // v = keep v s
  __device__ __forceinline__ void drop(int c, float (&v)[4]) const {
    if (mask.cut != 0) apply_mask(mask, key, t, per, c, v);
  }
  // the gradient of n, and branch normalised (branch itself without a norm)
  __device__ __forceinline__ void post(int c, float (&dn)[4], float (&bh)[4]) const {
    float g[4];
    d(c, dn);
    drop(c, dn);
    param4(a.gate != nullptr ? a.gate + gate_row(t, a.gate_rows) * a.D : nullptr, c, a.D, 1.0f, g);
    load_part(static_cast<const BT*>(a.branch) + t * a.ldb + c, a.D - c, bmean, bh);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      dn[e] *= g[e];
      bh[e] = (bh[e] - bmean) * brstd;
    }
  }
};

// The four sums of every row, [4][T]: c1 and c2 of N_pre', then of N_post'.
template <typename ST, typename BT>
__global__ __launch_bounds__(kWide) void block_grad_sums_kernel(const emb_block_norm_grad_args a, DropMask mask,
                                                                float* __restrict__ out) {
  __shared__ float2 red[2][kWaves];
  Sums sums{red, 0};
  const int D = a.D, step = kWide * 4, c_first = static_cast<int>(threadIdx.x) * 4;
  const float fD = static_cast<float>(D);
  const uint64_t key = mask_key(mask);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    GradRow<ST, BT> row(a, mask, key, t);
    float s1 = 0.0f, s2 = 0.0f, u[4], v[4], w[4];
    if (a.pre_stats != nullptr) {
      for (int c = c_first; c < D; c += step) {
        row.pre(c, u, v);
        param4(a.pre_weight, c, D, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s1 += u[e] * w[e];
          s2 += u[e] * w[e] * v[e];
        }
      }
      sums(s1, s2);
      row.c1 = s1 / fD;
      row.c2 = s2 / fD;
    }
    s1 = s2 = 0.0f;
    if (a.post_stats != nullptr) {
      for (int c = c_first; c < D; c += step) {
        row.post(c, u, v);
        param4(a.post_weight, c, D, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s1 += c + e < D ? u[e] * w[e] : 0.0f;
          s2 += c + e < D ? u[e] * w[e] * v[e] : 0.0f;
        }
      }
      sums(s1, s2);
    }
    if (threadIdx.x == 0) {
      out[t] = row.c1;
      out[a.T + t] = row.c2;
      out[2 * static_cast<int64_t>(a.T) + t] = s1 / fD;
      out[3 * static_cast<int64_t>(a.T) + t] = s2 / fD;
    }
  }
}

template <typename ST, typename BT>
__global__ __launch_bounds__(kWide) void block_grad_rows_kernel(const emb_block_norm_grad_args a, DropMask mask,
                                                                const float* __restrict__ in) {
  const int D = a.D, step = kWide * 4;
  const uint64_t key = mask_key(mask);
  const float alpha = static_cast<float>(a.alpha);
  for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
    GradRow<ST, BT> row(a, mask, key, t);
    row.c1 = in[t];
    row.c2 = in[a.T + t];
    const float c3 = in[2 * static_cast<int64_t>(a.T) + t], c4 = in[3 * static_cast<int64_t>(a.T) + t];
    for (int c = static_cast<int>(threadIdx.x) * 4; c < D; c += step) {
      float d[4], dn[4], bh[4], w[4];
      row.d(c, d);
      row.post(c, dn, bh);
      if (a.dx != nullptr) {
#pragma unroll
        for (int e = 0; e < 4; ++e) d[e] *= alpha;
        store_part(static_cast<ST*>(a.dx) + t * a.lddx + c, D - c, d);
      }
      if (a.dbranch != nullptr) {
        if (a.post_stats != nullptr) {
          param4(a.post_weight, c, D, 1.0f, w);
#pragma unroll
          for (int e = 0; e < 4; ++e) dn[e] = row.brstd * (dn[e] * w[e] - c3 - bh[e] * c4);
        }
        store_part(static_cast<BT*>(a.dbranch) + t * a.lddb + c, D - c, dn);
      }
    }
  }
}

// Column sums: a lane has four columns of the rows begin + blockIdx.y, + gridDim.y, ... of the range.
// part [gridDim.y][5][D]: dpre_weight, dpre_bias, dpost_weight, dpost_bias, dgate of all rows.
template <typename ST, typename BT>
__device__ __forceinline__ void column_step(const GradRow<ST, BT>& row, int c, int D, float (&s)[5][4]) {
  float u[4], v[4], w[4], b[4];
  if (row.a.pre_stats != nullptr) {
    row.pre(c, u, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[0][e] += u[e] * v[e];
      s[1][e] += u[e];
    }
  }
  row.post(c, u, v);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    s[2][e] += u[e] * v[e];
    s[3][e] += u[e];
  }
  row.d(c, u);
  if (row.a.post_stats != nullptr) {
    param4(row.a.post_weight, c, D, 1.0f, w);
    param4(row.a.post_bias, c, D, 0.0f, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] * w[e] + b[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) u[e] *= v[e];
  row.drop(c, u);
#pragma unroll
  for (int e = 0; e < 4; ++e) s[4][e] += u[e];
}
template <typename ST, typename BT>
__global__ __launch_bounds__(kThreads) void block_columns_kernel(const emb_block_norm_grad_args a, DropMask mask,
                                                                 const float* __restrict__ in, float* __restrict__ part) {
  const int c = (static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x)) * 4;
  if (c >= a.D) return;
  const uint64_t key = mask_key(mask);
  float s[5][4] = {};
  for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
    GradRow<ST, BT> row(a, mask, key, t);
    row.c1 = in[t];
    row.c2 = in[a.T + t];
    column_step(row, c, a.D, s);
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) store_part(part + (static_cast<int64_t>(blockIdx.y) * 5 + k) * a.D + c, a.D - c, s[k]);
}
// dgate where rows have gates of their own: every workgroup takes whole groups of rows.
template <typename ST, typename BT>
__global__ __launch_bounds__(kThreads) void block_gates_kernel(const emb_block_norm_grad_args a, DropMask mask,
                                                               const float* __restrict__ in) {
  const int c = (static_cast<int>(blockIdx.x) * kThreads + static_cast<int>(threadIdx.x)) * 4;
  if (c >= a.D) return;
  const uint64_t key = mask_key(mask);
  const int64_t gates = (a.T + a.gate_rows - 1) / a.gate_rows;
  for (int64_t g = blockIdx.y; g < gates; g += gridDim.y) {
    float s[5][4] = {};
    const int64_t end = min(static_cast<int64_t>(a.T), (g + 1) * a.gate_rows);
    for (int64_t t = g * a.gate_rows; t < end; ++t) {
      GradRow<ST, BT> row(a, mask, key, t);
      row.c1 = in[t];
      row.c2 = in[a.T + t];
      column_step(row, c, a.D, s);
    }
    store_part(a.dgate + g * a.D + c, a.D - c, s[4]);
  }
}

// dgate of the groups that several places share: the sum of their pieces in row order, one element per lane.
struct Pieces {
  const float* p;
  int64_t T, gate_rows, run;
  float* dgate;
};
constexpr int kSum = 32;
__device__ __forceinline__ void sum_pieces(const Pieces& s, int D, int64_t i) {
  const int64_t g = i / D, c = i % D;
  if (g * s.gate_rows >= s.T) return;
  const int64_t first = g * s.gate_rows / s.run, last = (min(s.T, (g + 1) * s.gate_rows) - 1) / s.run;
  if (first == last) return;
  // the first place may have had a group before this one, the others begin in it
  float v = s.p[(first * 2 + (first * s.run / s.gate_rows == g ? 0 : 1)) * D + c];
#pragma unroll 8
  for (int64_t p = first + 1; p <= last; ++p) v += s.p[p * 2 * D + c];
  s.dgate[i] = v;
}

// out_k[c] = sum over the partial rows of part[p][k][c], in their order; a workgroup takes 32 columns, its lanes'
// groups every 32nd partial row.  The workgroups from `sums` on: dgate from its pieces, in the same launch, since each of
// the two is a wait for memory and little else (9999 rows of 300, 33 to a gate: 5.8 and 4.7 us as launches of their own).
struct Outs {
  float* p[5];
};
__global__ __launch_bounds__(kSum* kSum) void block_sum_kernel(const float* __restrict__ part, int nparts, int D,
                                                               int64_t first, int64_t sums, Outs outs, Pieces pieces) {
  __shared__ float red[kSum][kSum + 1];
  const int col = static_cast<int>(threadIdx.x) % kSum, g = static_cast<int>(threadIdx.x) / kSum;
  if (first + blockIdx.x >= sums) {
    sum_pieces(pieces, D, (first + blockIdx.x - sums) * (kSum * kSum) + threadIdx.x);
    return;
  }
  const int64_t c0 = (first + blockIdx.x) * kSum, n = 5 * static_cast<int64_t>(D), c = c0 + col;
  float s = 0.0f;
  if (c < n) {
#pragma unroll 16
    for (int p = g; p < nparts; p += kSum) s += part[p * n + c];
  }
  red[g][col] = s;
  __syncthreads();
  s = group_sum<kSum>(red[col][g]);
  const int64_t o = c0 + g;
  if (col == 0 && o < n) {
    float* out = outs.p[o / D];
    if (out != nullptr) out[o % D] = s;
  }
}

constexpr int kParts = 256;  // partial rows of the column sums at most
int parts_for(int64_t T) { return static_cast<int>(T < 16 * kParts ? (T + 15) / 16 : kParts); }

// How the backward pass of rows in registers is spread; elements of a lane, per vector and at most.
constexpr int kNarrow = 16;  // forward
struct GradPlan {
  RowPlan row;
  bool fits;
  int places, blocks;  // rows at once per workgroup; workgroups
  int64_t run;         // rows of a place, where groups of rows have gates
  bool shared;         // some group is split over places
};
GradPlan plan_grad(int64_t T, int D, int64_t gate_rows, int E) {
  GradPlan p{};
  p.row = plan_row(D, E, kGradMost);
  p.fits = p.row.waves > 0 && p.row.nv * E <= kGradMost;
  if (!p.fits || T == 0) return p;
  p.places = grad_threads(p.row.waves) / (p.row.waves * p.row.lanes);
  const int64_t b = (T + p.places - 1) / p.places, most = p.row.nv * E <= kGradFew ? 768 : 512;
  p.blocks = static_cast<int>(b < most ? b : most);
  if (gate_rows > 0) {
    const int64_t all = static_cast<int64_t>(p.blocks) * p.places;
    p.run = (T + all - 1) / all;
    if (gate_rows <= p.run) p.run = (p.run + gate_rows - 1) / gate_rows * gate_rows;
    p.blocks = static_cast<int>((T + p.run * p.places - 1) / (p.run * p.places));
    p.shared = p.run % gate_rows != 0;
  }
  return p;
}

struct Work {
  float *sums, *part, *pieces;
};
size_t carve(char* base, int64_t T, int D, const GradPlan& p, Work& w) {
  Carver c{base};
  w.sums = w.pieces = nullptr;
  if (!p.fits) {
    w.sums = c.take<float>(4 * T);
    w.part = c.take<float>(static_cast<size_t>(parts_for(T)) * 5 * D);
  } else {
    w.part = c.take<float>(static_cast<size_t>(p.blocks) * 5 * D);
    if (p.shared) w.pieces = c.take<float>(static_cast<size_t>(p.blocks) * p.places * 2 * D);
  }
  return c.size();
}

// The column sums (columns), and dgate of the groups that places share (pieces.p).
void sum_parts(const emb_block_norm_grad_args& a, const float* part, int nparts, bool columns, bool gate,
               const Pieces& pieces, hipStream_t stream) {
  const Outs outs{{a.dpre_weight, a.dpre_bias, a.dpost_weight, a.dpost_bias, gate ? a.dgate : nullptr}};
  // a launch holds less than 2^32 threads
  const int64_t sums = columns ? (5 * static_cast<int64_t>(a.D) + kSum - 1) / kSum : 0;
  const int64_t gates = pieces.p != nullptr ? (a.T + a.gate_rows - 1) / a.gate_rows : 0;
  const int64_t blocks = sums + (gates * a.D + kSum * kSum - 1) / (kSum * kSum);
  for (int64_t first = 0; first < blocks; first += kMaxBlocks)
    block_sum_kernel<<<grid_for(blocks - first, kMaxBlocks), kSum * kSum, 0, stream>>>(part, nparts, a.D, first, sums, outs,
                                                                                       pieces);
}

template <typename ST, typename BT, int kE>
void grad_call(const emb_block_norm_grad_args& a, const DropMask& mask, hipStream_t stream) {
  const bool gates = a.dgate != nullptr && a.gate_rows > 0, gate = a.dgate != nullptr && !gates;
  const bool columns = gate || a.dpre_weight != nullptr || a.dpre_bias != nullptr || a.dpost_weight != nullptr ||
                       a.dpost_bias != nullptr;
  const GradPlan plan = plan_grad(a.T, a.D, gates ? a.gate_rows : 0, kE);
  Work w;
  carve(static_cast<char*>(a.workspace), a.T, a.D, plan, w);
  int nparts = 0;
  if (a.T > 0 && plan.fits) {
    nparts = plan.blocks;
    with_shape<kE, kGradMost>(plan.row, [&](auto L, auto NV, auto W) {
      if constexpr (NV.value * kE <= kGradMost) {
        const auto kernel = gates ? block_grad_kernel<ST, BT, kE, L.value, NV.value, W.value, true>
                                  : block_grad_kernel<ST, BT, kE, L.value, NV.value, W.value, false>;
        kernel<<<nparts, grad_threads(W.value), 0, stream>>>(a, mask, plan.run, columns ? w.part : nullptr, w.pieces);
      }
    });
  } else if (a.T > 0) {
    nparts = parts_for(a.T);
    const unsigned across = static_cast<unsigned>((a.D + 4 * kThreads - 1) / (4 * kThreads));
    block_grad_sums_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask, w.sums);
    // the sums first: dx may be written over dh, dbranch over dy
    if (columns) block_columns_kernel<ST, BT><<<dim3(across, nparts), kThreads, 0, stream>>>(a, mask, w.sums, w.part);
    if (gates)
      block_gates_kernel<ST, BT><<<dim3(across, grid_for((a.T + a.gate_rows - 1) / a.gate_rows, 16384)), kThreads, 0,
                                   stream>>>(a, mask, w.sums);
    if (a.dx != nullptr || a.dbranch != nullptr)
      block_grad_rows_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask, w.sums);
  }
  sum_parts(a, w.part, nparts, columns, gate, Pieces{w.pieces, a.T, a.gate_rows, plan.run, a.dgate}, stream);
}

template <typename ST, typename BT, int kE>
void block_call(const emb_block_norm_args& a, const DropMask& mask, hipStream_t stream) {
  const RowPlan pl = plan_row(a.D, kE, kNarrow);
  if (pl.waves == 0) {
    block_loop_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask);
    return;
  }
  with_shape<kE, kNarrow>(pl, [&](auto L, auto NV, auto W) {
    const int64_t rows = W.value > 1 ? 1 : kThreads / L.value;
    for (int64_t begin = 0; begin < a.T; begin += rows * kMaxBlocks)
      block_kernel<ST, BT, kE, L.value, NV.value, W.value>
          <<<grid_for((a.T - begin + rows - 1) / rows, kMaxBlocks), W.value > 1 ? W.value * kWave : kThreads, 0, stream>>>(
              a, mask, begin);
  });
}

}  // namespace

hipError_t launch_block_norm(const BlockArgs& b, hipStream_t stream) {
  const emb_block_norm_args& a = *b.a;
  if (a.T == 0) return hipSuccess;
  if (a.stream_dtype == EMB_BF16)
    block_call<bf16, bf16, 8>(a, b.mask, stream);
  else
    a.dtype == EMB_BF16 ? block_call<float, bf16, 4>(a, b.mask, stream) : block_call<float, float, 4>(a, b.mask, stream);
  return hipGetLastError();
}

size_t block_norm_grad_workspace_bytes(int64_t T, int D, int64_t gate_rows) {
  size_t most = 0;
  for (const int64_t rows : {int64_t{0}, gate_rows < T ? gate_rows : T})
    for (const int E : {4, 8}) {
      Work w;
      const size_t n = carve(nullptr, T, D, plan_grad(T, D, rows, E), w);
      if (n > most) most = n;
    }
  return most;
}

hipError_t launch_block_norm_grad(const BlockGradArgs& b, hipStream_t stream) {
  const emb_block_norm_grad_args& a = *b.a;
  if (a.stream_dtype == EMB_BF16)
    grad_call<bf16, bf16, 8>(a, b.mask, stream);
  else
    a.dtype == EMB_BF16 ? grad_call<float, bf16, 4>(a, b.mask, stream) : grad_call<float, float, 4>(a, b.mask, stream);
  return hipGetLastError();
}

}  // namespace emb
