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
#include "vec.h"

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
constexpr int kThreads = 256;
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

// out_k[c] = sum over the partial rows of part[p][k][c], in their order; a workgroup takes 32 columns, its lanes'
// groups every 32nd partial row.
struct Outs {
  float* p[5];
};
constexpr int kSum = 32;
__global__ __launch_bounds__(kSum* kSum) void block_sum_kernel(const float* __restrict__ part, int nparts, int D,
                                                               int64_t first, Outs outs) {
  __shared__ float red[kSum][kSum + 1];
  const int col = static_cast<int>(threadIdx.x) % kSum, g = static_cast<int>(threadIdx.x) / kSum;
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

struct Work {
  float *sums, *part;
};
size_t carve(char* base, int64_t T, int D, Work& w) {
  Carver c{base};
  w.sums = c.take<float>(4 * T);
  w.part = c.take<float>(static_cast<size_t>(parts_for(T)) * 5 * D);
  return c.size();
}

void sum_parts(const emb_block_norm_grad_args& a, const float* part, int nparts, bool gate, hipStream_t stream) {
  const Outs outs{{a.dpre_weight, a.dpre_bias, a.dpost_weight, a.dpost_bias, gate ? a.dgate : nullptr}};
  // a launch holds less than 2^32 threads
  const int64_t blocks = (5 * static_cast<int64_t>(a.D) + kSum - 1) / kSum;
  for (int64_t first = 0; first < blocks; first += kMaxBlocks)
    block_sum_kernel<<<grid_for(blocks - first, kMaxBlocks), kSum * kSum, 0, stream>>>(part, nparts, a.D, first, outs);
}

template <typename ST, typename BT>
void grad_call(const emb_block_norm_grad_args& a, const DropMask& mask, hipStream_t stream) {
  Work w;
  carve(static_cast<char*>(a.workspace), a.T, a.D, w);
  const bool gates = a.dgate != nullptr && a.gate_rows > 0, gate = a.dgate != nullptr && !gates;
  const bool columns = gate || a.dpre_weight != nullptr || a.dpre_bias != nullptr || a.dpost_weight != nullptr ||
                       a.dpost_bias != nullptr;
  const int nparts = parts_for(a.T);
  const unsigned across = static_cast<unsigned>((a.D + 4 * kThreads - 1) / (4 * kThreads));
  if (a.T > 0) {
    block_grad_sums_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask, w.sums);
    // the sums first: dx may be written over dh, dbranch over dy
    if (columns) block_columns_kernel<ST, BT><<<dim3(across, nparts), kThreads, 0, stream>>>(a, mask, w.sums, w.part);
    if (gates)
      block_gates_kernel<ST, BT><<<dim3(across, grid_for((a.T + a.gate_rows - 1) / a.gate_rows, 16384)), kThreads, 0,
                                   stream>>>(a, mask, w.sums);
    if (a.dx != nullptr || a.dbranch != nullptr)
      block_grad_rows_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask, w.sums);
  }
  if (columns) sum_parts(a, w.part, a.T > 0 ? nparts : 0, gate, stream);
}

template <typename ST, typename BT>
void block_call(const emb_block_norm_args& a, const DropMask& mask, hipStream_t stream) {
  block_loop_kernel<ST, BT><<<grid_for(a.T, kMaxBlocks), kWide, 0, stream>>>(a, mask);
}

}  // namespace

hipError_t launch_block_norm(const BlockArgs& b, hipStream_t stream) {
  const emb_block_norm_args& a = *b.a;
  if (a.T == 0) return hipSuccess;
  if (a.stream_dtype == EMB_BF16)
    block_call<bf16, bf16>(a, b.mask, stream);
  else
    a.dtype == EMB_BF16 ? block_call<float, bf16>(a, b.mask, stream) : block_call<float, float>(a, b.mask, stream);
  return hipGetLastError();
}

size_t block_norm_grad_workspace_bytes(int64_t T, int D, int64_t) {
  Work w;
  return carve(nullptr, T, D, w);
}

hipError_t launch_block_norm_grad(const BlockGradArgs& b, hipStream_t stream) {
  const emb_block_norm_grad_args& a = *b.a;
  if (a.stream_dtype == EMB_BF16)
    grad_call<bf16, bf16>(a, b.mask, stream);
  else
    a.dtype == EMB_BF16 ? grad_call<float, bf16>(a, b.mask, stream) : grad_call<float, float>(a, b.mask, stream);
  return hipGetLastError();
}

}  // namespace emb
