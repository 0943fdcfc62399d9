// AdamW over many tensors in one launch, with moments in 32 or in 8 bits
// (Kingma & Ba, Algorithm 1, with the decoupled decay of Loshchilov & Hutter).
//
//   g <- grad_scale g;  m <- b1 m + (1 - b1) g;  v <- b2 v + (1 - b2) g^2
//   w <- w - lr decay w;  w <- w - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)
//
// Bound by memory: every element of w, g, m, v is read once and of w, m, v (and
// the bf16 copy) written once.  A workgroup takes one chunk of kChunk elements
// of one tensor; the tensors' addresses ride in the kernel's arguments, so a
// call allocates and copies nothing and may be captured in a graph.
//
// 8-bit moments: m in e4m3, v in e5m2 (v spans twice the powers of two that m
// does, and needs no sign), with one scale per kQBlock elements, the power of
// two that keeps the block's largest value below the top of the type's range.
// A wave holds a block, so its largest value is one reduction over lanes.
// Moments change by a small part of themselves per step (b2 = 0.999: by 0.1 %,
// an eighth of a percent of what one code step is), so rounding to nearest
// would leave them where they are; they are rounded up with the probability of
// the part that is cut off, and so follow the moment on average.  A v that is
// not 0 never becomes 0: the update divides by its root.  The update itself
// takes the moments before they are rounded.
//
// Compiled without fused multiply-adds: the moments, and with them the codes,
// are then the same on every path and for every way of writing the formula.
#include "vec.h"
#include "launch.h"

namespace emb {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4096;
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

// The code of |x| in a float of kMant mantissa bits and exponent bias kBias;
// inv is the inverse of the block's scale, rnd 16 random bits.  Below the
// smallest normal value 2^(1 - kBias) the codes are evenly spaced: adding that
// value moves x into the range above, where they are spaced alike.
template <int kMant, int kBias, bool kNeverZero>
__device__ __forceinline__ uint32_t code8(float x, float inv, uint32_t rnd) {
  const float t = fabsf(x) * inv;
  const float low = __uint_as_float(static_cast<uint32_t>(128 - kBias) << 23);
  const bool under = t < low;
  const float t2 = under ? t + low : t;
  constexpr int kCut = 23 - kMant;
  const uint32_t r = (rnd << (kCut - 16)) + (1u << (kCut - 17));
  uint32_t c = ((__float_as_uint(t2) + r) >> kCut) - (static_cast<uint32_t>(under ? 128 - kBias : 127 - kBias) << kMant);
  if (kNeverZero) c = c == 0 && t > 0.0f ? 1u : c;
  return c;
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

__device__ __forceinline__ void update(float g, float& w, float& m, float& v, const AdamwCoeffs& c) {
  m = m * c.beta1 + g * c.one_minus_beta1;
  v = v * c.beta2 + g * g * c.one_minus_beta2;
  w = w - w * c.lr_decay;
  w = w - m / (sqrtf(v * c.inv_bc2) + c.eps) * c.step_size;
}

__device__ __forceinline__ bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

template <typename GT, bool k8, bool kCopy>
__global__ __launch_bounds__(kThreads) void adamw_kernel(const Batch b, int first, AdamwCoeffs cval,
                                                         const AdamwCoeffs* __restrict__ coeffs_dev,
                                                         const float* __restrict__ grad_scale, int32_t* status) {
  const AdamwCoeffs c = coeffs_dev != nullptr ? *coeffs_dev : cval;
  const int lane = static_cast<int>(lane_id());
  const int block = static_cast<int>(blockIdx.x);
  // the last tensor that starts at or before this workgroup
  const int k = uniform(__popcll(__ballot(b.start[lane] <= block)) - 1);
  const AdamwTensor& t = b.t[k];
  const int64_t n = t.n;
  const int64_t base = static_cast<int64_t>(block - b.start[k]) * kChunk;
  const float gs = grad_scale != nullptr ? *grad_scale : 1.0f;
  bool bad = false;
  float* scales = static_cast<float*>(t.scales);
  const int64_t nblocks = (n + kQBlock - 1) / kQBlock;
  const uint64_t key = k8 ? mix64(c.key + static_cast<uint64_t>(first + k + 1) * kGamma) : 0;
#pragma unroll
  for (int it = 0; it < kChunk / (kThreads * 4); ++it) {
    const int64_t i = base + (it * kThreads + static_cast<int>(threadIdx.x)) * 4;
    const int left = static_cast<int>(i + 4 <= n ? 4 : n - i);
    if (!k8 && left <= 0) break;
    float w[4], g[4], m[4], v[4];
    load_part(t.param + i, left, 0.0f, w);
    load_part(static_cast<const GT*>(t.grad) + i, left, 0.0f, g);
    if constexpr (!k8) {
      load_part(static_cast<const float*>(t.exp_avg) + i, left, 0.0f, m);
      load_part(static_cast<const float*>(t.exp_avg_sq) + i, left, 0.0f, v);
    } else {
      const int64_t q = base / kQBlock + uniform((it * kThreads + static_cast<int>(threadIdx.x)) / kWave);
      if (q >= nblocks) break;
      uint32_t mc = 0, vc = 0;
      const uint8_t* mp = static_cast<const uint8_t*>(t.exp_avg) + i;
      const uint8_t* vp = static_cast<const uint8_t*>(t.exp_avg_sq) + i;
      if (left >= 4) {
        mc = *reinterpret_cast<const words1_b*>(mp);
        vc = *reinterpret_cast<const words1_b*>(vp);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e < left) {
            mc |= static_cast<uint32_t>(mp[e]) << (8 * e);
            vc |= static_cast<uint32_t>(vp[e]) << (8 * e);
          }
        }
      }
      const float ms = scales[q], vs = scales[nblocks + q];
      m[0] = __builtin_amdgcn_cvt_f32_fp8(mc, 0) * ms;
      m[1] = __builtin_amdgcn_cvt_f32_fp8(mc, 1) * ms;
      m[2] = __builtin_amdgcn_cvt_f32_fp8(mc, 2) * ms;
      m[3] = __builtin_amdgcn_cvt_f32_fp8(mc, 3) * ms;
      v[0] = __builtin_amdgcn_cvt_f32_bf8(vc, 0) * vs;
      v[1] = __builtin_amdgcn_cvt_f32_bf8(vc, 1) * vs;
      v[2] = __builtin_amdgcn_cvt_f32_bf8(vc, 2) * vs;
      v[3] = __builtin_amdgcn_cvt_f32_bf8(vc, 3) * vs;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (grad_scale != nullptr) g[e] *= gs;
      update(g[e], w[e], m[e], v[e], c);
    }
    if constexpr (k8) {
      const int64_t q = base / kQBlock + uniform((it * kThreads + static_cast<int>(threadIdx.x)) / kWave);
      uint32_t mm = 0, vm = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        mm = e < left ? max(mm, __float_as_uint(m[e]) & 0x7FFFFFFFu) : mm;
        vm = e < left ? max(vm, __float_as_uint(v[e]) & 0x7FFFFFFFu) : vm;
      }
      mm = wave_max(mm);
      vm = wave_max(vm);
      float ms, vs, minv, vinv;
      block_scale<7>(mm, ms, minv);
      block_scale<14>(vm, vs, vinv);
      bad |= mm >= 0x7F800000u || vm >= 0x7F800000u;
      uint32_t mc = 0, vc = 0;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const uint64_t z = mix64(key + static_cast<uint64_t>((i + e) / 2 + 1) * kGamma);
#pragma unroll
        for (int o = 0; o < 2; ++o) {
          const uint32_t r = static_cast<uint32_t>(z >> (32 * o));
          mc |= (code8<3, 7, false>(m[e + o], minv, r & 0xFFFFu) | (__float_as_uint(m[e + o]) >> 24 & 0x80u)) << (8 * (e + o));
          vc |= code8<2, 15, true>(v[e + o], vinv, r >> 16) << (8 * (e + o));
        }
      }
      if (mm >= 0x7F800000u) mc = 0;  // the scale is NaN
      if (vm >= 0x7F800000u) vc = 0;
      uint8_t* mp = static_cast<uint8_t*>(t.exp_avg) + i;
      uint8_t* vp = static_cast<uint8_t*>(t.exp_avg_sq) + i;
      if (left >= 4) {
        *reinterpret_cast<words1_b*>(mp) = mc;
        *reinterpret_cast<words1_b*>(vp) = vc;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (e < left) {
            mp[e] = static_cast<uint8_t>(mc >> (8 * e));
            vp[e] = static_cast<uint8_t>(vc >> (8 * e));
          }
        }
      }
      if (lane == 0) {
        scales[q] = ms;
        scales[nblocks + q] = vs;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) bad |= e < left && (not_finite(m[e]) || not_finite(v[e]));
      store_part(static_cast<float*>(t.exp_avg) + i, left, m);
      store_part(static_cast<float*>(t.exp_avg_sq) + i, left, v);
    }
    store_part(t.param + i, left, w);
    if constexpr (kCopy) store_part(static_cast<bf16*>(t.copy) + i, left, w);
  }
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
  constexpr int64_t kMostBlocks = 1 << 23;  // workgroups of a launch (2^32 threads are too many)
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
