// C ABI entry points of the dense operators: host-side argument checks and the
// launches on the caller's stream.  Contract: include/emb.h.
#include <cmath>

#include "common.h"
#include "launch.h"

namespace {

constexpr int64_t kMaxV = (int64_t{1} << 31) - 1;

int launch_status(hipError_t e) { return e == hipSuccess ? EMB_OK : EMB_ERR_LAUNCH; }

bool bad_dtype(int32_t t) { return t != EMB_F32 && t != EMB_BF16; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
size_t elem_bytes(int32_t t) { return t == EMB_BF16 ? 2 : 4; }

bool bad_row_dims(int32_t T, int32_t D) { return T < 0 || T >= (1 << 30) || D < 1 || D >= (1 << 28); }

}  // namespace

extern "C" {

int emb_layer_norm(const void* x, int32_t x_dtype, int64_t ldx, const int32_t* ids, int64_t V, int32_t T, int32_t D,
                   const float* weight, const float* bias, double eps, void* y, int32_t y_dtype, int64_t ldy,
                   float* mean, float* rstd, int32_t* dev_status, void* stream) {
  if (bad_row_dims(T, D) || bad_dtype(x_dtype) || bad_dtype(y_dtype) || ldx < 0 || ldy < D || !(eps >= 0.0) ||
      !std::isfinite(eps) || (ids != nullptr && (V < 1 || V > kMaxV)))
    return EMB_ERR_INVALID_ARG;
  if (T == 0) return EMB_OK;
  if (!x || !y || !mean || !rstd) return EMB_ERR_INVALID_ARG;
  if (misaligned(x, elem_bytes(x_dtype)) || misaligned(y, elem_bytes(y_dtype)) || misaligned(weight, 4) ||
      misaligned(bias, 4))
    return EMB_ERR_INVALID_ARG;
  const emb::NormArgs a{x,   ldx, ids,  V,    T,          D,          weight, bias, eps, y,
                        ldy, mean, rstd, dev_status, x_dtype == EMB_BF16, y_dtype == EMB_BF16};
  return launch_status(emb::launch_norm(a, static_cast<hipStream_t>(stream)));
}

size_t emb_layer_norm_backward_workspace_bytes(int32_t T, int32_t D) {
  return bad_row_dims(T, D) ? 0 : emb::norm_grad_workspace_bytes(T, D);
}

int emb_layer_norm_backward(const void* dy, int32_t dy_dtype, int64_t lddy, const void* x, int32_t x_dtype,
                            int64_t ldx, const int32_t* ids, int64_t V, int32_t T, int32_t D, const float* weight,
                            const float* mean, const float* rstd, void* dx, int64_t lddx, float* dweight,
                            float* dbias, void* workspace, size_t workspace_bytes, int32_t* dev_status,
                            void* stream) {
  if (bad_row_dims(T, D) || bad_dtype(x_dtype) || bad_dtype(dy_dtype) || ldx < 0 || lddy < 0 ||
      (dx != nullptr && lddx < D) || (ids != nullptr && (V < 1 || V > kMaxV)))
    return EMB_ERR_INVALID_ARG;
  if (dx == nullptr && dweight == nullptr && dbias == nullptr) return EMB_ERR_INVALID_ARG;
  if (T > 0 && (!dy || !x || !mean || !rstd)) return EMB_ERR_INVALID_ARG;
  if (misaligned(x, elem_bytes(x_dtype)) || misaligned(dy, elem_bytes(dy_dtype)) ||
      misaligned(dx, elem_bytes(dy_dtype)) || misaligned(weight, 4) || misaligned(dweight, 4) || misaligned(dbias, 4))
    return EMB_ERR_INVALID_ARG;
  const bool params = dweight != nullptr || dbias != nullptr;
  if (params && T > 0 && (!workspace || misaligned(workspace, 256))) return EMB_ERR_INVALID_ARG;
  if (params && T > 0 && workspace_bytes < emb::norm_grad_workspace_bytes(T, D)) return EMB_ERR_WORKSPACE;
  const emb::NormGradArgs a{dy,   lddy, x,  ldx,  ids,     V,     T,         D,          weight,
                            mean, rstd, dx, lddx, dweight, dbias, workspace, dev_status, x_dtype == EMB_BF16,
                            dy_dtype == EMB_BF16};
  return launch_status(emb::launch_norm_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
