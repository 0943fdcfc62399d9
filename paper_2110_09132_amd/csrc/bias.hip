// Relative position bias by buckets, and its gradient.
//
//   out[h][i][j] = table[bucket_of[clamp(j - (q0 + i), -R, R) + R]][h]
//   dtable[b][h] = sum over n, i, j with that bucket of grad[n][h][i][j]
//
// Every diagonal of a head's (i, j) plane holds one value, so a plane is one
// line of Q + K - 1 values.  Forward: bound by the writes of the planes.  A
// workgroup forms the part of the line that its tile needs in LDS; a thread
// keeps one vector of columns and goes down the rows, and from one row to the
// next its vector shifts by one element: one LDS read for 16 bytes written.
// Backward: bound by the reads of the gradients.  A thread keeps kE
// neighbouring diagonals and goes down the rows with its column moving along;
// the sums stay in registers, need no atomics and have a fixed order.
#include <type_traits>

#include "vec.h"
#include "launch.h"

namespace emb {
namespace {

constexpr int kThreads = 256;

template <typename T>
constexpr int vec_elems() {
  return 16 / sizeof(T);
}

// Place in bucket_of of the position difference rel.
__device__ __forceinline__ int64_t place(int64_t rel, int64_t R) { return (rel < -R ? -R : rel > R ? R : rel) + R; }

// A tile of `rows` rows and tx * kE columns of one head; the workgroup's
// threads are tx columns' vectors by kThreads / tx groups of rows.
template <typename T>
__global__ __launch_bounds__(kThreads) void bias_kernel(const float* __restrict__ table, int num_buckets, int H,
                                                        const int32_t* __restrict__ bucket_of, int64_t R, int Q, int K,
                                                        int64_t q0, T* __restrict__ out, int64_t ldq, int64_t ldh,
                                                        int log2tx, int rows, int32_t* status) {
  constexpr int kE = vec_elems<T>();
  extern __shared__ float line[];  // line[u]: the value where (j - j0) - (i - i0) + rows - 1 == u
  const int tx = 1 << log2tx;
  const int h = static_cast<int>(blockIdx.y);
  const int ntx = (K + tx * kE - 1) / (tx * kE);
  const int j0 = static_cast<int>(blockIdx.x % ntx) * tx * kE;
  const int i0 = static_cast<int>(blockIdx.x / ntx) * rows;
  const int n = min(tx * kE, K - j0) + rows - 1;
  bool bad = false;
  for (int u = static_cast<int>(threadIdx.x); u < n; u += kThreads) {
    const int64_t rel = static_cast<int64_t>(j0) - i0 + (u - (rows - 1)) - q0;
    const int32_t b = bucket_of[place(rel, R)];
    bad |= b >= num_buckets;
    line[u] = b < 0 ? -__builtin_inff() : b < num_buckets ? table[static_cast<size_t>(b) * H + h] : 0.0f;
  }
  __syncthreads();
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_BUCKET_OUT_OF_RANGE);
  const int c = (static_cast<int>(threadIdx.x) & (tx - 1)) * kE;
  const int per = rows >> (8 - log2tx);  // rows of this thread (kThreads == 2^8)
  const int l0 = (static_cast<int>(threadIdx.x) >> log2tx) * per;
  if (j0 + c >= K) return;
  float v[kE];
#pragma unroll
  for (int e = 0; e < kE - 1; ++e) v[e] = line[min(c + e + 1 - l0 + rows - 1, n - 1)];
  T* o = out + static_cast<int64_t>(h) * ldh + static_cast<int64_t>(i0 + l0) * ldq + j0 + c;
  for (int l = l0; l < l0 + per && i0 + l < Q; ++l, o += ldq) {
#pragma unroll
    for (int e = kE - 1; e > 0; --e) v[e] = v[e - 1];
    v[0] = line[c - l + rows - 1];
    store_part(o, K - j0 - c, v);
  }
}

// The sums of the diagonals of `rows` rows: part[h][tile][u] with
// u = j - (i - i0) + rows - 1, u < K + rows - 1.  Diagonals without a bucket
// are not read where a thread has only such, and count as nothing elsewhere.
template <typename T>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const T* __restrict__ grad, int N, int64_t ldn,
                                                             int64_t ldh, int64_t ldq, int Q, int K, int64_t q0,
                                                             const int32_t* __restrict__ bucket_of, int64_t R,
                                                             int num_buckets, int rows, float* __restrict__ part,
                                                             int32_t* status) {
  constexpr int kE = vec_elems<T>();
  const int nu = K + rows - 1;
  const int chunks = (nu + kThreads * kE - 1) / (kThreads * kE);
  const int tile = static_cast<int>(blockIdx.x) / chunks;
  const int u0 = ((static_cast<int>(blockIdx.x) % chunks) * kThreads + static_cast<int>(threadIdx.x)) * kE;
  const int h = static_cast<int>(blockIdx.y);
  const int i0 = tile * rows;
  const int nr = min(rows, Q - i0);
  bool bad = false;
  bool used[kE], any = false;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    used[e] = false;
    if (u0 + e < nu) {
      const int32_t b = bucket_of[place(static_cast<int64_t>(u0 + e - (rows - 1)) - i0 - q0, R)];
      bad |= b >= num_buckets;
      used[e] = b >= 0 && b < num_buckets;
    }
    any |= used[e];
  }
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_BUCKET_OUT_OF_RANGE);
  if (u0 >= nu) return;
  float acc[kE] = {};
  if (any) {
    const int c0 = u0 - (rows - 1);  // column of the thread's first diagonal at local row 0
    for (int n = 0; n < N; ++n) {
      const T* g = grad + n * ldn + h * ldh + static_cast<int64_t>(i0) * ldq;
#pragma unroll 4
      for (int l = 0; l < nr; ++l, g += ldq) {
        const int c = c0 + l;
        float v[kE];
        if (c >= 0 && c + kE <= K) {
          load_vec(g + c, v);
        } else {
#pragma unroll
          for (int e = 0; e < kE; ++e) v[e] = c + e >= 0 && c + e < K ? widen(g[c + e]) : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < kE; ++e) acc[e] += v[e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < kE; ++e) acc[e] = used[e] ? acc[e] : 0.0f;
  store_part(part + (static_cast<size_t>(h) * (gridDim.x / chunks) + tile) * nu + u0, nu - u0, acc);
}

// dtable[b][h]: the sums of the diagonals whose bucket is b, one workgroup per (b, h).
__global__ __launch_bounds__(kThreads) void bias_fold_kernel(const float* __restrict__ part, int tiles, int rows,
                                                             int K, int64_t q0, const int32_t* __restrict__ bucket_of,
                                                             int64_t R, int H, float* __restrict__ dtable) {
  __shared__ float red[kThreads / kWave];
  const int b = static_cast<int>(blockIdx.x), h = static_cast<int>(blockIdx.y);
  const int nu = K + rows - 1;
  float s = 0.0f;
  for (int tile = 0; tile < tiles; ++tile) {
    const float* p = part + (static_cast<size_t>(h) * tiles + tile) * nu;
    for (int u = static_cast<int>(threadIdx.x); u < nu; u += kThreads) {
      const int64_t rel = static_cast<int64_t>(u - (rows - 1)) - static_cast<int64_t>(tile) * rows - q0;
      s += bucket_of[place(rel, R)] == b ? p[u] : 0.0f;
    }
  }
  s = group_sum<kWave>(s);
  if (lane_id() == 0) red[threadIdx.x / kWave] = s;
  __syncthreads();
  if (threadIdx.x == 0) dtable[static_cast<size_t>(b) * H + h] = (red[0] + red[1]) + (red[2] + red[3]);
}

constexpr int kGradRows = 16;
int grad_rows(int Q) { return Q < kGradRows ? (Q < 1 ? 1 : Q) : kGradRows; }
int grad_tiles(int Q) { return (Q + grad_rows(Q) - 1) / grad_rows(Q); }

template <typename T>
void bias_call(const BiasArgs& a, hipStream_t stream) {
  constexpr int kE = vec_elems<T>();
  int log2tx = 0;
  while ((1 << log2tx) * kE < a.K && log2tx < 8) ++log2tx;
  const int groups = kThreads >> log2tx;
  int per = (a.Q + groups - 1) / groups;  // rows per thread
  per = per < 32 ? per : 32;
  const int rows = groups * per;
  const int64_t tiles = static_cast<int64_t>((a.K + (kE << log2tx) - 1) / (kE << log2tx)) * ((a.Q + rows - 1) / rows);
  const size_t lds = (static_cast<size_t>(kE << log2tx) + rows) * sizeof(float);
  bias_kernel<T><<<dim3(static_cast<unsigned>(tiles), a.H), kThreads, lds, stream>>>(
      a.table, a.num_buckets, a.H, a.bucket_of, a.R, a.Q, a.K, a.q0, static_cast<T*>(a.out), a.ldq, a.ldh, log2tx,
      rows, a.status);
}

template <typename T>
void bias_grad_call(const BiasGradArgs& a, hipStream_t stream) {
  constexpr int kE = vec_elems<T>();
  const int rows = grad_rows(a.Q), tiles = a.N > 0 && a.K > 0 && a.Q > 0 ? grad_tiles(a.Q) : 0;
  float* part = static_cast<float*>(a.workspace);
  if (tiles > 0) {
    const int64_t chunks = (static_cast<int64_t>(a.K) + rows - 1 + kThreads * kE - 1) / (kThreads * kE);
    bias_grad_kernel<T><<<dim3(static_cast<unsigned>(chunks * tiles), a.H), kThreads, 0, stream>>>(
        static_cast<const T*>(a.grad), a.N, a.ldn, a.ldh, a.ldq, a.Q, a.K, a.q0, a.bucket_of, a.R, a.num_buckets, rows,
        part, a.status);
  }
  bias_fold_kernel<<<dim3(a.num_buckets, a.H), kThreads, 0, stream>>>(part, tiles, rows, a.K, a.q0, a.bucket_of, a.R,
                                                                       a.H, a.dtable);
}

}  // namespace

hipError_t launch_bias(const BiasArgs& a, hipStream_t stream) {
  if (a.Q == 0 || a.K == 0) return hipSuccess;
  a.out_bf16 ? bias_call<bf16>(a, stream) : bias_call<float>(a, stream);
  return hipGetLastError();
}

size_t bias_grad_workspace_bytes(int N, int H, int Q, int K) {
  if (N == 0 || Q == 0 || K == 0) return 256;
  Carver c{nullptr};
  c.take<float>(static_cast<size_t>(H) * grad_tiles(Q) * (static_cast<size_t>(K) + grad_rows(Q) - 1));
  return c.size();
}

hipError_t launch_bias_grad(const BiasGradArgs& a, hipStream_t stream) {
  a.grad_bf16 ? bias_grad_call<bf16>(a, stream) : bias_grad_call<float>(a, stream);
  return hipGetLastError();
}

}  // namespace emb
