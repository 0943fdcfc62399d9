// Dropout from a counter-based generator: y = residual + keep x / (1 - q).
//
// Bound by memory: x (and the residual) are read once, y is written once, and
// the mask costs one draw of SplitMix64 per four elements.
#include "dropout.h"
#include "vec.h"

namespace emb {
namespace {

constexpr int kThreads = 256;

// L lanes per row, kThreads / L rows per workgroup, kE elements per lane and
// step; a workgroup takes the next rows in memory and ends.
template <typename T, int kE>
__global__ __launch_bounds__(kThreads) void dropout_kernel(const T* x, int64_t ldx, const T* residual, int64_t ldr,
                                                           int64_t begin, int64_t rows, int D, int log2_lanes, DropMask mask,
                                                           T* y, int64_t ldy) {
  const int lanes = 1 << log2_lanes, lane = static_cast<int>(threadIdx.x) & (lanes - 1);
  const int64_t t = begin + (static_cast<int64_t>(blockIdx.x) << (8 - log2_lanes)) + (threadIdx.x >> log2_lanes);
  if (t >= rows) return;
  const uint64_t key = mask_key(mask);
  const int64_t per = (static_cast<int64_t>(D) + 3) / 4;
  const T* xr = x + t * ldx;
  T* yr = y + t * ldy;
  const int64_t step = static_cast<int64_t>(lanes) * kE;
  for (int64_t c = static_cast<int64_t>(blockIdx.y) * step + lane * kE; c < D; c += gridDim.y * step) {
    const int n = static_cast<int>(min(D - c, static_cast<int64_t>(kE)));
    float v[kE], r[kE];
    load_part<true>(xr + c, n, 0.0f, v);
    if (residual != nullptr) load_part<true>(residual + t * ldr + c, n, 0.0f, r);
    if (mask.cut != 0) apply_mask(mask, key, t, per, static_cast<int>(c), v);
    if (residual != nullptr) {
#pragma unroll
      for (int e = 0; e < kE; ++e) v[e] += r[e];
    }
    store_part<true>(yr + c, n, v);
  }
}

template <typename T, int kE>
void dropout_call(const DropoutArgs& a, hipStream_t stream) {
  int log2_lanes = 0;
  while (log2_lanes < 8 && (static_cast<int64_t>(kE) << log2_lanes) < a.D) ++log2_lanes;
  const int64_t rows = kThreads >> log2_lanes;
  const int64_t steps = (a.D + (static_cast<int64_t>(kE) << log2_lanes) - 1) / (static_cast<int64_t>(kE) << log2_lanes);
  const unsigned across = static_cast<unsigned>(steps < 1024 ? steps : 1024);
  const int64_t most = kMaxBlocks / across;
  for (int64_t b = 0; b < a.T; b += rows * most)
    dropout_kernel<T, kE><<<dim3(grid_for((a.T - b + rows - 1) / rows, most), across), kThreads, 0, stream>>>(
        static_cast<const T*>(a.x), a.ldx, static_cast<const T*>(a.residual), a.ldr, b, a.T, a.D, log2_lanes, a.mask,
        static_cast<T*>(a.y), a.ldy);
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, hipStream_t stream) {
  if (a.T == 0) return hipSuccess;
  a.is_bf16 ? dropout_call<bf16, 8>(a, stream) : dropout_call<float, 4>(a, stream);
  return hipGetLastError();
}

}  // namespace emb
