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
// Backward: bound by the reads of the gradients.  A thread walks along the
// diagonals; the sums stay in registers, need no atomics and have a fixed order.
#include <algorithm>

#include "vec.h"
#include "launch.h"
#include "places.h"

namespace emb {
namespace {

constexpr int kThreads = 256;

template <typename T>
constexpr int vec_elems() {
  return 16 / sizeof(T);
}

// A tile of `rows` rows and `width` columns of one head; the workgroup's threads
// are tx columns' vectors by kThreads / tx groups of rows.  Tiles of about
// kTileBytes and of whole rows up to kTileCols, so that the workgroups write one
// front through memory and a line that two rows share is written by one of them;
// at least kFewRows rows, so that forming the line costs little.  Measured (16
// planes of 2048 x 2048): fp32, 2 whole rows 42 us (6.4 TB/s; a fill reaches
// 6.7), 4 half rows 46, 4 whole rows 51; bf16, 4 rows 25 to 29, 2 rows 42, 8 rows
// 27; planes of 2047 x 2047 fp32: 4 half rows 62 us, whole rows 54.
constexpr int kTileBytes = 16384;
template <typename T>
constexpr int kTileCols = sizeof(T) == 4 ? 4096 : 2048;
template <typename T>
constexpr int kFewRows = sizeof(T) == 4 ? 2 : 4;
template <typename T>
__global__ __launch_bounds__(kThreads) void bias_kernel(const float* __restrict__ table, int num_buckets, int H,
                                                        const int32_t* __restrict__ bucket_of, int R, int Q, int K,
                                                        int64_t q0, T* __restrict__ out, int64_t ldq, int64_t ldh,
                                                        int log2tx, int width, int rows, int first_row,
                                                        int32_t* status) {
  constexpr int kE = vec_elems<T>();
  // line[u]: the value where (j - j0) - (i - i0) + rows - 1 + kE == u (the last
  // vector of a row is moved back so that it ends there, up to kE before j0)
  extern __shared__ float line[];
  const int tx = 1 << log2tx;
  const int h = static_cast<int>(blockIdx.y);
  const int ntx = (K + width - 1) / width;
  const int j0 = static_cast<int>(blockIdx.x % ntx) * width;
  const int i0 = first_row + static_cast<int>(blockIdx.x / ntx) * rows;
  const int n = min(width, K - j0) + rows - 1 + kE;
  const int32_t base = base_of(static_cast<int64_t>(j0) - i0 - (rows - 1) - kE - q0, R);
  const int paired = kE + rows - min(rows, Q - i0);  // line[u] from here on has a pair in the tile's rows
  bool bad = false;
  constexpr int kAhead = 4;  // values in flight per thread; reads past the tile's end read its last value
  for (int u0 = static_cast<int>(threadIdx.x); u0 < n; u0 += kAhead * kThreads) {
    int32_t b[kAhead];
    float v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) b[k] = bucket_of[place(base, min(u0 + k * kThreads, n - 1), R)];
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      v[k] = table[static_cast<size_t>(min(max(b[k], 0), num_buckets - 1)) * H + h];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int u = u0 + k * kThreads;
      bad |= u >= paired && b[k] >= num_buckets;
      if (u < n) line[u] = b[k] < 0 ? -__builtin_inff() : b[k] < num_buckets ? v[k] : 0.0f;
    }
  }
  __syncthreads();
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_BUCKET_OUT_OF_RANGE);
  const int per = rows >> (8 - log2tx);  // rows of this thread (kThreads == 2^8)
  const int l0 = (static_cast<int>(threadIdx.x) >> log2tx) * per;
  const int nr = min(per, Q - i0 - l0);
  T* o = out + static_cast<int64_t>(h) * ldh + static_cast<int64_t>(i0 + l0) * ldq + j0;
  for (int c0 = (static_cast<int>(threadIdx.x) & (tx - 1)) * kE; c0 < width && j0 + c0 < K; c0 += tx * kE) {
    const int c = K >= kE ? min(c0, K - j0 - kE) : c0;
    const float* at = line + c - l0 + rows - 1 + kE;  // where column c of row l0 stands
    float v[kE];
#pragma unroll
    for (int e = 0; e < kE - 1; ++e) v[e] = at[K >= kE ? e + 1 : min(e + 1, K - 1)];
    for (int l = 0; l < nr; ++l) {
#pragma unroll
      for (int e = kE - 1; e > 0; --e) v[e] = v[e - 1];
      v[0] = at[-l];
      if (K >= kE)
        store_vec(o + l * ldq + c, v);
      else
        store_part(o + l * ldq + c, K, v);
    }
  }
}

// How the gradient's work is split: a workgroup takes `rows` queries and
// kThreads bands of columns of one head, for n_per batch entries, and leaves the
// sums of its diagonals per place of bucket_of.
struct GradPlan {
  int rows;      // a multiple of 8
  int threads;   // bands per workgroup
  int chunks;    // workgroups side by side over a tile's bands
  int tiles;     // tiles of rows
  int n_per, nz; // batch entries per workgroup, workgroups over the batch
  int window;    // places per workgroup
  __host__ __device__ int blocks() const { return tiles * chunks * nz; }
};

// Place range of a workgroup: its window starts at the place of its first
// diagonal (the difference `first`), moved so that it ends inside bucket_of.
__device__ __forceinline__ int64_t window_start(int64_t first, int64_t R, int window) {
  const int64_t last = 2 * R + 1 - window;
  return max(min(first + R, last), static_cast<int64_t>(0));
}

// Sum over a workgroup of up to kThreads threads, in all of them.
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* red) {
  a = group_sum<kWave>(a);
  b = group_sum<kWave>(b);
  if (lane_id() == 0) red[threadIdx.x / kWave] = make_float2(a, b);
  __syncthreads();
  float2 s = red[0];
  for (int w = 1; w < static_cast<int>(blockDim.x) / kWave; ++w) {
    s.x += red[w].x;
    s.y += red[w].y;
  }
  return s;
}

// A thread walks down the diagonal in squares of kE x kE elements: every load is
// an aligned vector where the rows are, and all squares of a thread lie on the
// same 2 kE - 1 diagonals, whose sums stay in registers.  Neighbouring threads
// share kE - 1 diagonals, joined in LDS.
template <typename T>
__global__ __launch_bounds__(kThreads) void bias_grad_kernel(const T* __restrict__ grad, int N, int64_t ldn,
                                                             int64_t ldh, int64_t ldq, int Q, int K, int64_t q0,
                                                             const int32_t* __restrict__ bucket_of, int64_t R,
                                                             GradPlan pl, float* __restrict__ part) {
  constexpr int kE = vec_elems<T>();
  constexpr int kD = 2 * kE - 1;
  __shared__ float line[kThreads * kE + kE - 1];
  __shared__ float2 red[kThreads / kWave];
  const int t = static_cast<int>(threadIdx.x);
  const int tile = static_cast<int>(blockIdx.x) / pl.chunks, chunk = static_cast<int>(blockIdx.x) % pl.chunks;
  const int h = static_cast<int>(blockIdx.y);
  const int i0 = tile * pl.rows;
  const int nr = min(pl.rows, Q - i0);
  const int64_t cb0 = static_cast<int64_t>(chunk) * pl.threads * kE - (pl.rows - kE);
  const int64_t cb = cb0 + t * kE;  // the thread's first column in the tile's first rows
  const int64_t first = cb0 - (kE - 1) - i0 - q0;  // difference of line[0]
  float acc[kD] = {};
  bool any = false;
#pragma unroll
  for (int d = 0; d < kD; ++d) any |= bucket_of[place(base_of(first, static_cast<int32_t>(R)), t * kE + d, R)] >= 0;
  const auto add = [&](const Vec<T, kE>(&v)[kE]) {
#pragma unroll
    for (int l = 0; l < kE; ++l)
#pragma unroll
      for (int e = 0; e < kE; ++e) acc[e - l + kE - 1] += v[l][e];
  };
  const int l0 = cb < 0 ? static_cast<int>(-cb) : 0;  // first local row whose square is in the plane
  if (any && cb < K && l0 < nr) {
    const int c0 = static_cast<int>(cb + l0);
    const int n0 = static_cast<int>(blockIdx.z) * pl.n_per, n1 = min(N, n0 + pl.n_per);
    const T* plane = grad + n0 * ldn + h * ldh + static_cast<int64_t>(i0 + l0) * ldq + c0;
    const int whole = min(nr - l0, K - c0) / kE;  // squares that the plane's and the tile's end leave whole
    const int lw = whole * kE, rows_left = nr - l0 - lw, cols_left = K - c0 - lw;
    for (int n = n0; n < n1; ++n, plane += ldn) {
      const T* g = plane;
      for (int k = 0; k < whole; ++k, g += kE * ldq + kE) {
        Vec<T, kE> v[kE];
#pragma unroll
        for (int l = 0; l < kE; ++l) v[l].template load<true>(g + l * ldq, kE);
        add(v);
      }
      if (rows_left > 0 && cols_left > 0) {
        // the square that is cut: what is past its last row and column is read from there, and left out
        float v[kE][kE];
        if (cols_left >= kE) {
#pragma unroll
          for (int l = 0; l < kE; ++l) load_vec(g + min(l, rows_left - 1) * ldq, v[l]);
        } else {
#pragma unroll
          for (int l = 0; l < kE; ++l)
#pragma unroll
            for (int e = 0; e < kE; ++e) v[l][e] = widen(g[min(l, rows_left - 1) * ldq + min(e, cols_left - 1)]);
        }
#pragma unroll
        for (int l = 0; l < kE; ++l)
#pragma unroll
          for (int e = 0; e < kE; ++e) acc[e - l + kE - 1] += l < rows_left && e < cols_left ? v[l][e] : 0.0f;
      }
    }
  }
  // line[x]: the sum of the diagonal with difference first + x
#pragma unroll
  for (int x = 0; x < kE; ++x) line[t * kE + kE - 1 + x] = acc[kE - 1 + x];
  if (t == 0) {
#pragma unroll
    for (int d = 0; d < kE - 1; ++d) line[d] = acc[d];
  }
  __syncthreads();
  if (t > 0) {
#pragma unroll
    for (int d = 0; d < kE - 1; ++d) line[t * kE + d] += acc[d];
  }
  __syncthreads();
  // the ends of bucket_of take all diagonals beyond them
  const int64_t n = static_cast<int64_t>(pl.threads) * kE + kE - 1;
  const int64_t below = R == 0 ? n : min(max(-R - first + 1, static_cast<int64_t>(0)), n);
  const int64_t above = R == 0 ? n : min(max(R - first, static_cast<int64_t>(0)), n);
  float a = 0.0f, b = 0.0f;
  for (int64_t x = t; x < below; x += pl.threads) a += line[x];
  for (int64_t x = above + t; x < n; x += pl.threads) b += line[x];
  const float2 ends = block_sum2(a, b, red);
  const int64_t start = window_start(first, R, pl.window);
  float* out = part + ((static_cast<size_t>(h) * gridDim.z + blockIdx.z) * gridDim.x + blockIdx.x) * pl.window;
  for (int w = t; w < pl.window; w += pl.threads) {
    const int64_t p = start + w, x = p - R - first;
    float v = x >= 0 && x < n ? line[x] : 0.0f;
    if (p == 2 * R) v = ends.y;
    if (p == 0) v = ends.x;
    out[w] = bucket_of[p] >= 0 ? v : 0.0f;
  }
}

// Place at which the window of a head's workgroup k starts.
template <typename T>
__device__ __forceinline__ int64_t windows_start(const GradPlan& pl, int64_t q0, int64_t R, int k) {
  constexpr int kE = vec_elems<T>();
  const int x = k % (pl.tiles * pl.chunks);
  const int64_t first = static_cast<int64_t>(x % pl.chunks) * pl.threads * kE - (pl.rows - kE) - (kE - 1) -
                        static_cast<int64_t>(x / pl.chunks) * pl.rows - q0;
  return window_start(first, R, pl.window);
}

// dtable from the windows in one launch, a workgroup per head: for up to
// kFewWindows windows that each hold all places, and up to kFewPlaces of those
// (128 windows of 16 heads: 5 us, 8 to 11 us in two launches; 384 windows: 6 and
// 11 us).  Its waves take every kFoldWaves-th window.
constexpr int kFoldWaves = 16;
constexpr int kFewPlaces = 512;
constexpr int kFewWindows = 512;
__global__ __launch_bounds__(kFoldWaves* kWave) void bias_fold_kernel(const float* __restrict__ part, int nblocks,
                                                                      int window,
                                                                      const int32_t* __restrict__ bucket_of, int p0,
                                                                      int places, int num_buckets, int H,
                                                                      float* __restrict__ dtable, int32_t* status) {
  constexpr int kPer = kFewPlaces / kWave;
  __shared__ float red[kFoldWaves][kFewPlaces];
  __shared__ int32_t bucket[kFewPlaces];
  const int t = static_cast<int>(threadIdx.x), lane = static_cast<int>(lane_id());
  const int wave = uniform(t / kWave);
  const int h = static_cast<int>(blockIdx.x);
  const float* in = part + static_cast<size_t>(h) * nblocks * window + p0;
  int at[kPer];  // lanes past the last place read the last
#pragma unroll
  for (int i = 0; i < kPer; ++i) at[i] = min(i * kWave + lane, places - 1);
  float s[kPer] = {};
#pragma unroll 2
  for (int k = wave; k < nblocks; k += kFoldWaves) {
    const float* w = in + static_cast<size_t>(k) * window;
#pragma unroll
    for (int i = 0; i < kPer; ++i) s[i] += w[at[i]];
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) red[wave][i * kWave + lane] = s[i];
  int32_t mine = -1;
  if (t < places) mine = bucket_of[p0 + t];
  if (__any(mine >= num_buckets) && lane == 0) raise_flag(status, EMB_DEV_BUCKET_OUT_OF_RANGE);
  __syncthreads();
  if (t < kFewPlaces) {
    float v = red[0][t];
#pragma unroll
    for (int i = 1; i < kFoldWaves; ++i) v += red[i][t];
    red[0][t] = v;
    bucket[t] = mine;
  }
  __syncthreads();
  for (int64_t b = wave; b < num_buckets; b += kFoldWaves) {
    float v = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) v += bucket[i * kWave + lane] == b ? red[0][i * kWave + lane] : 0.0f;
    v = group_sum<kWave>(v);
    if (lane == 0) dtable[static_cast<size_t>(b) * H + h] = v;
  }
}

// Else in two: the sums of the windows per place, for the `places` places from p0
// on, the ones that occur, a workgroup per head and 64 places (the launch's first
// takes place `first` of them);
template <typename T>
__global__ __launch_bounds__(kFoldWaves* kWave) void bias_places_kernel(
    const float* __restrict__ part, GradPlan pl, int64_t q0, const int32_t* __restrict__ bucket_of, int64_t R,
    int64_t p0, int places, int first, int num_buckets, float* __restrict__ sums, int32_t* status) {
  __shared__ float red[kFoldWaves][kWave];
  const int lane = static_cast<int>(lane_id());
  const int wave = uniform(static_cast<int>(threadIdx.x) / kWave);
  const int h = static_cast<int>(blockIdx.y);
  const int64_t c = static_cast<int64_t>(first) + static_cast<int>(blockIdx.x) * kWave + lane;
  const int64_t p = p0 + min(c, static_cast<int64_t>(places) - 1);
  const int nblocks = pl.blocks();
  const float* in = part + static_cast<size_t>(h) * nblocks * pl.window;
  float s = 0.0f;
  if (pl.window == 2 * R + 1) {  // every window holds all places
#pragma unroll 16
    for (int k = wave; k < nblocks; k += kFoldWaves) s += in[static_cast<size_t>(k) * pl.window + p];
  } else {
#pragma unroll 8
    for (int k = wave; k < nblocks; k += kFoldWaves) {
      const int64_t w = p - windows_start<T>(pl, q0, R, k);
      const float v = in[static_cast<size_t>(k) * pl.window + (w < 0 || w >= pl.window ? 0 : w)];
      s += w < 0 || w >= pl.window ? 0.0f : v;
    }
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave > 0) return;
  bool bad = false;
  if (c < places) {
#pragma unroll
    for (int i = 1; i < kFoldWaves; ++i) s += red[i][lane];
    sums[static_cast<size_t>(h) * places + c] = s;
    bad = bucket_of[p0 + c] >= num_buckets;
  }
  if (__any(bad) && lane == 0) raise_flag(status, EMB_DEV_BUCKET_OUT_OF_RANGE);
}

// then the places' sums per bucket, a wave per bucket from `first` on.
__global__ __launch_bounds__(kThreads) void bias_buckets_kernel(const float* __restrict__ sums,
                                                                const int32_t* __restrict__ bucket_of, int places,
                                                                int first, int num_buckets, int H,
                                                                float* __restrict__ dtable) {
  constexpr int kAhead = 8;
  const int h = static_cast<int>(blockIdx.y);
  const int64_t b = static_cast<int64_t>(first) + static_cast<int>(blockIdx.x) * (kThreads / kWave) +
                    static_cast<int>(threadIdx.x) / kWave;
  if (b >= num_buckets) return;
  const float* in = sums + static_cast<size_t>(h) * places;
  float s = 0.0f;
  for (int c0 = static_cast<int>(lane_id()); c0 < places; c0 += kAhead * kWave) {
    int32_t bk[kAhead];
    float v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int c = min(c0 + k * kWave, places - 1);
      bk[k] = bucket_of[c];
      v[k] = in[c];
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) s += c0 + k * kWave < places && bk[k] == b ? v[k] : 0.0f;
  }
  s = group_sum<kWave>(s);
  if (lane_id() == 0) dtable[static_cast<size_t>(b) * H + h] = s;
}

// Tiles of few rows keep the workgroups' reads close together in memory, and a
// tile of kE rows needs no band beyond the columns (K / kE bands: 128 or 256 for
// the usual widths, whole waves).  Measured: 8 x 16 x 1024 x 1024 bf16, 8 rows
// 45 us (6.0 TB/s; reads alone reach 6.6), 16 rows 46, 128 rows 50; 2 x 16 x
// 2048 x 2048 bf16 causal, 38, 43, 51; 16 x 2048 x 2048 fp32, 8 and 16 rows 51,
// 128 rows 47.  A head's windows are added up by few workgroups, so the tiles grow to leave
// kGoodWindows of them as long as there are workgroups enough, and kMostWindows
// in any case.
constexpr int64_t kManyBlocks = 1024;
constexpr int64_t kManyWaves = 2048;
constexpr int64_t kGoodWindows = 256, kMostWindows = 2048;
GradPlan plan_grad(int N, int H, int Q, int K, int E) {
  GradPlan pl;
  const int64_t groups = (static_cast<int64_t>(K) + E - 1) / E;
  const auto shape = [&](int rows) {
    const int64_t bands = groups + rows / E - 1;
    pl.rows = rows;
    pl.chunks = static_cast<int>((bands + kThreads - 1) / kThreads);
    pl.threads = static_cast<int>((bands + pl.chunks - 1) / pl.chunks + kWave - 1) / kWave * kWave;
    pl.tiles = static_cast<int>((static_cast<int64_t>(Q) + rows - 1) / rows);
  };
  int rows = E == 4 && Q > 8 ? 16 : 8;
  shape(rows);
  if (rows > 8 && static_cast<int64_t>(pl.tiles) * pl.chunks * H * N < kManyBlocks) shape(rows = 8);
  // narrow planes: more rows per workgroup fill its lanes
  while (rows < Q && groups + rows / E - 1 < kWave && static_cast<int64_t>(pl.tiles) * H * N >= 2 * kManyBlocks)
    shape(rows *= 2);
  while (rows < Q) {
    const int64_t windows = static_cast<int64_t>(pl.tiles) * pl.chunks;
    if (windows <= kMostWindows && (windows <= kGoodWindows || windows * H * N < 2 * kManyBlocks)) break;
    shape(rows *= 2);
  }
  // workgroups over the batch until the chip has kManyWaves
  const int64_t waves = static_cast<int64_t>(pl.tiles) * pl.chunks * H * (pl.threads / kWave);
  const int64_t nz = std::min<int64_t>((kManyWaves + waves - 1) / waves, N);
  pl.n_per = static_cast<int>((N + nz - 1) / nz);
  pl.nz = (N + pl.n_per - 1) / pl.n_per;
  pl.window = pl.threads * E + E - 1;
  return pl;
}

template <typename T>
void bias_call(const BiasArgs& a, hipStream_t stream) {
  constexpr int kE = vec_elems<T>();
  int log2tx = 0;
  while ((1 << log2tx) * kE < a.K && log2tx < 8) ++log2tx;
  const int groups = kThreads >> log2tx;
  const int vecs = kE << log2tx;
  // a tile of few rows is kept narrow, to have more of them
  const int width = a.Q < kFewRows<T> ? vecs : std::max(vecs, std::min((a.K + vecs - 1) / vecs * vecs, kTileCols<T>));
  const int most = std::max(kFewRows<T>, std::min(kTileBytes / (groups * width * static_cast<int>(sizeof(T))), 8));
  const int per = std::min((a.Q + groups - 1) / groups, most);  // rows per thread
  const int rows = groups * per;
  const int64_t across = (a.K + width - 1) / width, down = (a.Q + rows - 1) / rows;  // tiles
  const size_t lds = (static_cast<size_t>(width) + rows + kE) * sizeof(float);
  // a launch holds less than 2^32 threads: as many whole rows of tiles as kMaxBlocks takes (`across` is at most 2^20)
  const int64_t most_down = kMaxBlocks / across;
  for (int64_t i = 0; i < down; i += most_down)
    bias_kernel<T><<<dim3(static_cast<unsigned>(across) * grid_for(down - i, most_down), a.H), kThreads, lds, stream>>>(
        a.table, a.num_buckets, a.H, a.bucket_of, a.R, a.Q, a.K, a.q0, static_cast<T*>(a.out), a.ldq, a.ldh, log2tx,
        width, rows, static_cast<int>(i * rows), a.status);
}

template <typename T>
void bias_grad_call(const BiasGradArgs& a, hipStream_t stream) {
  constexpr int kE = vec_elems<T>();
  const bool pairs = a.N > 0 && a.K > 0 && a.Q > 0;
  // the places that occur: those of the differences -(Q - 1) - q0 .. K - 1 - q0
  const auto place_of = [&](int64_t rel) { return (rel < -a.R ? -a.R : rel > a.R ? a.R : rel) + a.R; };
  const int64_t p0 = pairs ? place_of(-(static_cast<int64_t>(a.Q) - 1) - a.q0) : 0;
  const int places = pairs ? static_cast<int>(place_of(a.K - 1 - a.q0) - p0 + 1) : 0;
  Carver c{static_cast<char*>(a.workspace)};
  GradPlan pl{};
  float* part = nullptr;
  if (pairs) {
    pl = plan_grad(a.N, a.H, a.Q, a.K, kE);
    if (2 * static_cast<int64_t>(a.R) + 1 < pl.window) pl.window = 2 * a.R + 1;
    part = c.take<float>(static_cast<size_t>(a.H) * pl.blocks() * pl.window);
    bias_grad_kernel<T><<<dim3(pl.tiles * pl.chunks, a.H, pl.nz), pl.threads, 0, stream>>>(
        static_cast<const T*>(a.grad), a.N, a.ldn, a.ldh, a.ldq, a.Q, a.K, a.q0, a.bucket_of, a.R, pl, part);
  }
  if (pairs && pl.window == 2 * static_cast<int64_t>(a.R) + 1 && places <= kFewPlaces && pl.blocks() <= kFewWindows) {
    bias_fold_kernel<<<a.H, kFoldWaves * kWave, 0, stream>>>(part, pl.blocks(), pl.window, a.bucket_of,
                                                             static_cast<int>(p0), places, a.num_buckets, a.H,
                                                             a.dtable, a.status);
    return;
  }
  float* sums = c.take<float>(static_cast<size_t>(a.H) * places);
  // a launch holds less than 2^32 threads
  const auto launches = [](int64_t work, int64_t per, auto&& launch) {  // `per` of the work in a workgroup
    for (int64_t first = 0; first < work; first += per * kMaxBlocks)
      launch(grid_for((work - first + per - 1) / per, kMaxBlocks), static_cast<int>(first));
  };
  launches(places, kWave, [&](unsigned grid, int first) {
    bias_places_kernel<T><<<dim3(grid, a.H), kFoldWaves * kWave, 0, stream>>>(
        part, pl, a.q0, a.bucket_of, a.R, p0, places, first, a.num_buckets, sums, a.status);
  });
  launches(a.num_buckets, kThreads / kWave, [&](unsigned grid, int first) {
    bias_buckets_kernel<<<dim3(grid, a.H), kThreads, 0, stream>>>(sums, a.bucket_of + p0, places, first, a.num_buckets,
                                                                  a.H, a.dtable);
  });
}

}  // namespace

hipError_t launch_bias(const BiasArgs& a, hipStream_t stream) {
  if (a.Q == 0 || a.K == 0) return hipSuccess;
  a.out_bf16 ? bias_call<bf16>(a, stream) : bias_call<float>(a, stream);
  return hipGetLastError();
}

size_t bias_grad_workspace_bytes(int N, int H, int Q, int K) {
  if (N == 0 || Q == 0 || K == 0) return 256;
  size_t most = 0;
  for (const int E : {vec_elems<float>(), vec_elems<bf16>()}) {
    const GradPlan pl = plan_grad(N, H, Q, K, E);
    Carver c{nullptr};
    c.take<float>(static_cast<size_t>(H) * pl.blocks() * pl.window);
    c.take<float>(static_cast<size_t>(H) * (static_cast<size_t>(Q) + K));
    if (c.size() > most) most = c.size();
  }
  return most;
}

hipError_t launch_bias_grad(const BiasGradArgs& a, hipStream_t stream) {
  a.grad_bf16 ? bias_grad_call<bf16>(a, stream) : bias_grad_call<float>(a, stream);
  return hipGetLastError();
}

}  // namespace emb
