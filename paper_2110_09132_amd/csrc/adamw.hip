// AdamW over many tensors in one launch, with moments in 32 or in 8 bits
// (Kingma & Ba, Algorithm 1, with the decoupled decay of Loshchilov & Hutter).
//
//   g <- grad_scale g;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   w <- w - lr decay w;  w <- w - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every element of w, g, m, v is read once and of w, m, v (and
// the bf16 copy) written once.  A workgroup takes one chunk of kChunk elements
// of one tensor, one vector of 4 per lane, and ends: the workgroups then move
// through memory as one front (75.6 million elements, bf16 gradients and copies,
// 2.1 GB: chunks of 1024 353 us, 6.0 TB/s, of 2048 368 us, of 4096 388 us; with
// plain instead of streaming accesses 388 us).  The tensors' addresses ride in
// the kernel's arguments, so a call allocates and copies nothing and may be
// captured in a graph.
//
// 8-bit moments: m in e4m3, v in e5m2 (v spans twice the powers of two that m
// does, and needs no sign), with one scale per kQBlock elements, the power of
// two that keeps the block's largest value below the top of the type's range.
// A wave holds a block, so its largest value is one reduction over lanes.
// v changes by a small part of itself per step (b2 = 0.999: by 0.1 %, while
// neighbouring codes are 14 to 25 % apart), so rounding to nearest would leave
// it where it is; both are rounded up with the probability of
// the part that is cut off, and so follow the moment on average.  A v that is
// not 0 never becomes 0: the update divides by its root.  The update itself
// takes the moments before they are rounded.  The conversions are the
// hardware's, with its random rounding, since the instructions of a wave are
// what bounds the kernel (the same elements, 1.2 GB: 259 us with conversions in
// software and 451 vector instructions per wave; 236 us with 342 so, 5.1 TB/s
// under the profiler, 216 us in a loop of calls).  The root and the quotient,
// each rounded to nearest, are about 100 of the 342; the kernel for 32-bit
// moments has 206 instructions per wave with them and is bound by memory.
//
// Compiled without fused multiply-adds: the moments, and with them the codes,
// are then the same on every path and for every way of writing the formula.
#include "vec.h"
#include "launch.h"

namespace emb {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = kThreads * 4;
constexpr int kQBlock = 256;  // elements that share a scale: 64 lanes of 4
constexpr int kPerLaunch = 64;

struct Batch {
  AdamwTensor t[kPerLaunch];
  int32_t start[kPerLaunch];  // first workgroup of each tensor; INT32_MAX past the last
};

typedef uint32_t words1_b __attribute__((aligned(1), may_alias));  // 4 values of 8 bits

// SplitMix64's output function (Steele, Lea & Flood 2014).
__device__ __forceinline__ uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
constexpr uint64_t kGamma = 0x9E3779B97F4A7C15ull;

// Bits of |x|, which are ordered as the magnitudes are: kInfinity, above it NaN.
__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }
constexpr uint32_t kInfinity = 0x7F800000u;

__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max(x, dpp_move<0xB1, 0xf>(x));
  x = max(x, dpp_move<0x4E, 0xf>(x));
  x = max(x, dpp_move<0x141, 0xf>(x));
  x = max(x, dpp_move<0x140, 0xf>(x));
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(r[0], r[1]);
  const auto s = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(s[0], s[1]);
}

// Scale of a block whose largest magnitude has these bits: that value over the
// scale is in [2^kTop, 2^(kTop + 1)).  Its inverse is exact.
template <int kTop>
__device__ __forceinline__ void block_scale(uint32_t most, float& scale, float& inv) {
  const int e = static_cast<int>(most >> 23);
  const int field = max(e - kTop, 1);
  scale = e == 255 ? __builtin_nanf("") : __uint_as_float(static_cast<uint32_t>(field) << 23);
  inv = __uint_as_float(static_cast<uint32_t>(254 - field) << 23);
}

// The root and the quotient are rounded to nearest, subnormal operands too (the
// bare instruction for the root takes those as 0: v below 2^-126 then leaves a
// divisor of eps alone, and an infinite parameter where eps is 0).  A parameter
// that starts at 0 is its update, and the table's rows take theirs by the same
// operations.
__device__ __forceinline__ void update(float g, float& w, float& m, float& v, const AdamwCoeffs& c) {
  m = m * c.beta1 + g * c.one_minus_beta1;
  v = v * c.beta2 + g * g * c.one_minus_beta2;
  w = w - w * c.lr_decay;
  w = w - m / (sqrtf(v * c.inv_bc2) + c.eps) * c.step_size;
}

// Four 8-bit values of which the first n (4 or more: all) exist.
template <bool kFull>
__device__ __forceinline__ uint32_t load4(const void* p, int n) {
  if (kFull || n >= 4) return __builtin_nontemporal_load(static_cast<const words1_b*>(p));
  uint32_t x = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) x |= static_cast<uint32_t>(static_cast<const uint8_t*>(p)[e]) << (8 * e);
  return x;
}
template <bool kFull>
__device__ __forceinline__ void store4(void* p, int n, uint32_t x) {
  if (kFull || n >= 4) {
    __builtin_nontemporal_store(x, static_cast<words1_b*>(p));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) static_cast<uint8_t*>(p)[e] = static_cast<uint8_t>(x >> (8 * e));
}

// One chunk of a tensor: 4 elements per lane, a block of 8-bit moments per wave.
// kFull: all kChunk elements exist.  Returns whether a moment is not finite.
template <typename GT, bool k8, bool kCopy, bool kFull>
__device__ __forceinline__ bool chunk(const AdamwTensor& t, int64_t base, uint64_t key, const AdamwCoeffs& c, float gs) {
  const int at = static_cast<int>(threadIdx.x) * 4;
  const int left = kFull ? 4 : static_cast<int>(min(static_cast<int64_t>(kChunk), t.n - base)) - at;
  if (!k8 && left <= 0) return false;
  const int64_t i = base + at;
  float w[4], g[4], m[4], v[4];
  load_part<true>(t.param + i, left, 0.0f, w);
  load_part<true>(static_cast<const GT*>(t.grad) + i, left, 0.0f, g);
  if constexpr (!k8) {
    load_part<true>(static_cast<const float*>(t.exp_avg) + i, left, 0.0f, m);
    load_part<true>(static_cast<const float*>(t.exp_avg_sq) + i, left, 0.0f, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) update(g[e] * gs, w[e], m[e], v[e], c);
    store_part<true>(static_cast<float*>(t.exp_avg) + i, left, m);
    store_part<true>(static_cast<float*>(t.exp_avg_sq) + i, left, v);
    store_part<true>(t.param + i, left, w);
    if constexpr (kCopy) store_part<true>(static_cast<bf16*>(t.copy) + i, left, w);
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, max(magnitude(m[e]), magnitude(v[e])));
    return most >= kInfinity;
  } else {
    const int64_t nblocks = (t.n + kQBlock - 1) / kQBlock;
    const int64_t q = base / kQBlock + uniform(at / kQBlock);
    if (q >= nblocks) return false;  // the same for the whole wave
    uint8_t* mp = static_cast<uint8_t*>(t.exp_avg) + i;
    uint8_t* vp = static_cast<uint8_t*>(t.exp_avg_sq) + i;
    uint32_t mc = load4<kFull>(mp, left), vc = load4<kFull>(vp, left);
    const float ms0 = t.scales[q], vs0 = t.scales[nblocks + q];
    const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8(mc, true);
    const auto v01 = __builtin_amdgcn_cvt_pk_f32_bf8(vc, false), v23 = __builtin_amdgcn_cvt_pk_f32_bf8(vc, true);
    m[0] = m01[0] * ms0, m[1] = m01[1] * ms0, m[2] = m23[0] * ms0, m[3] = m23[1] * ms0;
    v[0] = v01[0] * vs0, v[1] = v01[1] * vs0, v[2] = v23[0] * vs0, v[3] = v23[1] * vs0;
    uint32_t mm = 0, vm = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      update(g[e] * gs, w[e], m[e], v[e], c);
      const bool live = kFull || e < left;
      mm = max(mm, live ? magnitude(m[e]) : 0u);
      vm = max(vm, live ? magnitude(v[e]) : 0u);
    }
    store_part<true>(t.param + i, left, w);
    if constexpr (kCopy) store_part<true>(static_cast<bf16*>(t.copy) + i, left, w);
    mm = wave_max(mm);
    vm = wave_max(vm);
    float ms, vs, minv, vinv;
    block_scale<7>(mm, ms, minv);
    block_scale<14>(vm, vs, vinv);
    // the numbers of the lane's two pairs of elements; the base's part is the same for all lanes
    uint64_t z = (key + static_cast<uint64_t>(base / 2 + 1) * kGamma) + static_cast<uint64_t>(at / 2) * kGamma;
    const uint64_t z01 = mix64(z), z23 = mix64(z + kGamma);
    const uint32_t r[4] = {static_cast<uint32_t>(z01), static_cast<uint32_t>(z01 >> 32), static_cast<uint32_t>(z23),
                           static_cast<uint32_t>(z23 >> 32)};
    // The conversions add the upper bits of their random number below the
    // mantissa and cut off: 20 of them for e4m3, 21 for e5m2, so a number of 16
    // bits and a half in the upper places is what the contract asks for.
    // 2^-16 is the smallest e5m2.
#define EMB_CODE(E)                                                                                              \
  mc = __builtin_amdgcn_cvt_sr_fp8_f32(m[E] * minv, static_cast<int>(r[E] << 16 | 0x8000u), mc, E);              \
  vc = __builtin_amdgcn_cvt_sr_bf8_f32(v[E] > 0.0f ? fmaxf(v[E] * vinv, 0x1p-16f) : 0.0f,                        \
                                       static_cast<int>((r[E] & 0xFFFF0000u) | 0x8000u), vc, E)
    EMB_CODE(0);
    EMB_CODE(1);
    EMB_CODE(2);
    EMB_CODE(3);
#undef EMB_CODE
    const bool mbad = mm >= kInfinity, vbad = vm >= kInfinity;  // the scale is NaN
    store4<kFull>(mp, left, mbad ? 0u : mc);
    store4<kFull>(vp, left, vbad ? 0u : vc);
    if (lane_id() == 0) {
      t.scales[q] = ms;
      t.scales[nblocks + q] = vs;
    }
    return mbad || vbad;
  }
}

template <typename GT, bool k8, bool kCopy>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Batch b, int first, AdamwCoeffs cval,
                                                         const AdamwCoeffs* __restrict__ coeffs_dev,
                                                         const float* __restrict__ grad_scale, int32_t* status) {
  const AdamwCoeffs c = coeffs_dev != nullptr ? *coeffs_dev : cval;
  const int block = static_cast<int>(blockIdx.x);
  // the last tensor that starts at or before this workgroup
  const int k = uniform(__popcll(__ballot(b.start[lane_id()] <= block)) - 1);
  const AdamwTensor& t = b.t[k];
  const int64_t base = static_cast<int64_t>(block - b.start[k]) * kChunk;
  const float gs = grad_scale != nullptr ? *grad_scale : 1.0f;
  const uint64_t key = k8 ? mix64(c.key + static_cast<uint64_t>(first + k + 1) * kGamma) : 0;
  const bool bad = base + kChunk <= t.n ? chunk<GT, k8, kCopy, true>(t, base, key, c, gs)
                                        : chunk<GT, k8, kCopy, false>(t, base, key, c, gs);
  if (__any(bad) && lane_id() == 0) raise_flag(status, EMB_DEV_NOT_FINITE);
}

template <typename GT, bool k8>
void adamw_call(const Batch& b, unsigned grid, int first, const AdamwArgs& a, hipStream_t stream) {
  if (a.copies)
    adamw_kernel<GT, k8, true><<<grid, kThreads, 0, stream>>>(b, first, a.c, a.coeffs_dev, a.grad_scale, a.status);
  else
    adamw_kernel<GT, k8, false><<<grid, kThreads, 0, stream>>>(b, first, a.c, a.coeffs_dev, a.grad_scale, a.status);
}

}  // namespace

hipError_t launch_adamw(const AdamwArgs& a, hipStream_t stream) {
  // workgroups of a launch, and of the largest tensor: 2^31 threads (2^32 are too many)
  constexpr int64_t kMostBlocks = 1 << 23;
  for (int k = 0; k < a.n;) {
    Batch b;
    int count = 0;
    int64_t blocks = 0;
    const int first = k;
    for (; k < a.n && count < kPerLaunch; ++k) {
      const int64_t chunks = (a.tensors[k].n + kChunk - 1) / kChunk;
      if (count > 0 && blocks + chunks > kMostBlocks) break;
      b.t[count] = a.tensors[k];
      b.start[count++] = static_cast<int32_t>(blocks);
      blocks += chunks;
    }
    for (int i = count; i < kPerLaunch; ++i) b.start[i] = INT32_MAX;
    if (blocks == 0) continue;
    const unsigned grid = static_cast<unsigned>(blocks);
    if (a.bits8)
      a.grad_bf16 ? adamw_call<bf16, true>(b, grid, first, a, stream) : adamw_call<float, true>(b, grid, first, a, stream);
    else
      a.grad_bf16 ? adamw_call<bf16, false>(b, grid, first, a, stream)
                  : adamw_call<float, false>(b, grid, first, a, stream);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace emb
