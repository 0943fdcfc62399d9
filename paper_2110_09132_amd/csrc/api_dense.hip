// C ABI entry points of the dense operators: host-side argument checks and the
// launches on the caller's stream.  Contract: include/emb.h.
#include <cmath>
#include <cstring>

#include "common.h"
#include "dropout.h"
#include "launch.h"

namespace {

constexpr int64_t kMaxV = (int64_t{1} << 31) - 1;

int launch_status(hipError_t e) { return e == hipSuccess ? EMB_OK : EMB_ERR_LAUNCH; }

bool bad_dtype(int32_t t) { return t != EMB_F32 && t != EMB_BF16; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
size_t elem_bytes(int32_t t) { return t == EMB_BF16 ? 2 : 4; }

bool bad_row_dims(int32_t T, int32_t D) { return T < 0 || T >= (1 << 30) || D < 1 || D >= (1 << 28); }

}  // namespace

namespace emb {

int adamw_coeffs(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step, uint64_t seed,
                 AdamwCoeffs* c) {
  AdamCoeffs a;
  const int st = adam_coeffs(lr, beta1, beta2, eps, step, &a);
  if (st != EMB_OK) return st;
  if (!(weight_decay >= 0.0) || !std::isfinite(weight_decay)) return EMB_ERR_INVALID_ARG;
  *c = AdamwCoeffs{a.beta1,   a.one_minus_beta1, a.beta2, a.one_minus_beta2,
                   a.step_size, a.inv_bc2,       a.eps,   static_cast<float>(lr * weight_decay),
                   mix64(seed + static_cast<uint64_t>(step) * kGamma)};
  return EMB_OK;
}

}  // namespace emb

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

namespace {
constexpr int64_t kMaxPos = int64_t{1} << 62;
bool bad_bias_dims(int32_t num_buckets, int32_t H, int32_t R, int32_t Q, int32_t K, int64_t q0) {
  return num_buckets < 1 || H < 1 || H > 65535 || R < 0 || R >= (1 << 30) || Q < 0 || Q >= (1 << 30) || K < 0 ||
         K >= (1 << 30) || q0 <= -kMaxPos || q0 >= kMaxPos;
}
}  // namespace

int emb_relative_bias(const float* table, int32_t num_buckets, int32_t H, const int32_t* bucket_of, int32_t R,
                      int32_t Q, int32_t K, int64_t q0, void* out, int32_t out_dtype, int64_t ldq, int64_t ldh,
                      int32_t* dev_status, void* stream) {
  if (bad_bias_dims(num_buckets, H, R, Q, K, q0) || bad_dtype(out_dtype)) return EMB_ERR_INVALID_ARG;
  if (Q == 0 || K == 0) return EMB_OK;
  if (ldq < K) return EMB_ERR_INVALID_ARG;
  // heads one after another, or side by side within each query's rows
  if (H > 1 && (ldh < K || ((ldh - K) / ldq < Q - 1 && (ldq - K) / ldh < H - 1))) return EMB_ERR_INVALID_ARG;
  if (!table || !bucket_of || !out) return EMB_ERR_INVALID_ARG;
  if (misaligned(table, 4) || misaligned(bucket_of, 4) || misaligned(out, elem_bytes(out_dtype)))
    return EMB_ERR_INVALID_ARG;
  const emb::BiasArgs a{table, num_buckets, H,   bucket_of, R,          Q, K, q0, out,
                        ldq,   ldh,         dev_status, out_dtype == EMB_BF16};
  return launch_status(emb::launch_bias(a, static_cast<hipStream_t>(stream)));
}

size_t emb_relative_bias_backward_workspace_bytes(int32_t N, int32_t H, int32_t Q, int32_t K) {
  if (N < 0 || bad_bias_dims(1, H, 0, Q, K, 0)) return 0;
  return emb::bias_grad_workspace_bytes(N, H, Q, K);
}

int emb_relative_bias_backward(const void* grad, int32_t grad_dtype, int32_t N, int32_t H, int32_t Q, int32_t K,
                               int64_t ldn, int64_t ldh, int64_t ldq, const int32_t* bucket_of, int32_t R,
                               int32_t num_buckets, int64_t q0, float* dtable, void* workspace,
                               size_t workspace_bytes, int32_t* dev_status, void* stream) {
  if (N < 0 || bad_bias_dims(num_buckets, H, R, Q, K, q0) || bad_dtype(grad_dtype) || ldn < 0 || ldh < 0 || ldq < 0)
    return EMB_ERR_INVALID_ARG;
  if (!bucket_of || !dtable || misaligned(bucket_of, 4) || misaligned(dtable, 4)) return EMB_ERR_INVALID_ARG;
  if (N > 0 && Q > 0 && K > 0) {
    if (!grad || misaligned(grad, elem_bytes(grad_dtype)) || !workspace || misaligned(workspace, 256))
      return EMB_ERR_INVALID_ARG;
    if (workspace_bytes < emb::bias_grad_workspace_bytes(N, H, Q, K)) return EMB_ERR_WORKSPACE;
  }
  const emb::BiasGradArgs a{grad, N,           H,  Q,      K,         ldn,        ldh, ldq, bucket_of,
                            R,    num_buckets, q0, dtable, workspace, dev_status, grad_dtype == EMB_BF16};
  return launch_status(emb::launch_bias_grad(a, static_cast<hipStream_t>(stream)));
}

int emb_relative_buckets(int32_t num_buckets, int32_t max_distance, int32_t causal, int32_t* out) {
  const int32_t m = causal != 0 ? num_buckets : num_buckets / 2;
  const int32_t e = m / 2;
  if (m < 2 || (causal == 0 && num_buckets % 2 != 0) || max_distance <= e || max_distance >= (1 << 30) || !out)
    return EMB_ERR_INVALID_ARG;
  const double per = (m - e) / std::log(static_cast<double>(max_distance) / e);
  for (int32_t r = -max_distance; r <= max_distance; ++r) {
    const int32_t n = r < 0 ? -r : r;
    int32_t b = n;
    if (n >= e) {
      // the small term puts distances that stand exactly at a bucket's start into it
      b = e + static_cast<int32_t>(std::log(static_cast<double>(n) / e) * per + 1e-9);
      b = b < m - 1 ? b : m - 1;
    }
    out[r + max_distance] = r <= 0 ? b : causal != 0 ? -1 : m + b;
  }
  return EMB_OK;
}

int emb_adamw_step(const emb_adamw_tensor* tensors, int32_t n_tensors, int32_t grad_dtype, int32_t state_bits,
                   double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                   uint64_t seed, const void* coeffs, const float* grad_scale, int32_t* dev_status, void* stream) {
  if (n_tensors < 0 || bad_dtype(grad_dtype) || (state_bits != 32 && state_bits != 8) || misaligned(coeffs, 16) ||
      misaligned(grad_scale, 4))
    return EMB_ERR_INVALID_ARG;
  emb::AdamwArgs a{};
  const int st = emb::adamw_coeffs(lr, beta1, beta2, eps, weight_decay, step, seed, &a.c);
  if (st != EMB_OK) return st;
  if (n_tensors > 0 && !tensors) return EMB_ERR_INVALID_ARG;
  const size_t state_bytes = state_bits == 8 ? 1 : 4;
  int with_copy = 0, without_copy = 0;
  for (int32_t k = 0; k < n_tensors; ++k) {
    const emb_adamw_tensor& t = tensors[k];
    if (t.n < 0 || t.n > (int64_t{1} << 33)) return EMB_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq || (state_bits == 8 && !t.scales))
      return EMB_ERR_INVALID_ARG;
    if (misaligned(t.param, 4) || misaligned(t.grad, elem_bytes(grad_dtype)) || misaligned(t.exp_avg, state_bytes) ||
        misaligned(t.exp_avg_sq, state_bytes) || (state_bits == 8 && misaligned(t.scales, 4)) || misaligned(t.copy, 2))
      return EMB_ERR_INVALID_ARG;
    ++(t.copy != nullptr ? with_copy : without_copy);
  }
  if (with_copy > 0 && without_copy > 0) return EMB_ERR_INVALID_ARG;
  a.tensors = tensors;
  a.n = n_tensors;
  a.coeffs_dev = static_cast<const emb::AdamwCoeffs*>(coeffs);
  a.grad_scale = grad_scale;
  a.status = dev_status;
  a.grad_bf16 = grad_dtype == EMB_BF16;
  a.bits8 = state_bits == 8;
  a.copies = with_copy > 0;
  return launch_status(emb::launch_adamw(a, static_cast<hipStream_t>(stream)));
}

int emb_adamw_coeffs(double lr, double beta1, double beta2, double eps, double weight_decay, int64_t step,
                     uint64_t seed, void* out) {
  if (out == nullptr) return EMB_ERR_INVALID_ARG;
  emb::AdamwCoeffs c;
  const int st = emb::adamw_coeffs(lr, beta1, beta2, eps, weight_decay, step, seed, &c);
  if (st != EMB_OK) return st;
  std::memset(out, 0, EMB_ADAMW_COEFFS_WORDS * 4);
  std::memcpy(out, &c, sizeof(c));
  return EMB_OK;
}

namespace {
// The mask of p and seed; false where p is out of range.
bool drop_mask(double p, uint64_t seed, const uint64_t* seed_dev, emb::DropMask* m) {
  if (!(p >= 0.0 && p < 1.0) || misaligned(seed_dev, 8)) return false;
  const double n = std::nearbyint(65536.0 * p);
  const uint32_t cut = n < 65535.0 ? static_cast<uint32_t>(n) : 65535u;
  *m = emb::DropMask{emb::mix64(seed), seed_dev, cut, static_cast<float>(65536.0 / (65536.0 - cut))};
  return true;
}
bool bad_f32(const void* p) { return misaligned(p, 4); }
}  // namespace

int emb_dropout(const void* x, int32_t dtype, int64_t ldx, int32_t T, int32_t D, double p, uint64_t seed,
                const uint64_t* seed_dev, const void* residual, int64_t ldr, void* y, int64_t ldy, void* stream) {
  emb::DropMask mask;
  if (bad_row_dims(T, D) || bad_dtype(dtype) || ldx < 0 || (residual != nullptr && ldr < 0) || ldy < D ||
      !drop_mask(p, seed, seed_dev, &mask))
    return EMB_ERR_INVALID_ARG;
  if (T == 0) return EMB_OK;
  const size_t e = elem_bytes(dtype);
  if (!x || !y || misaligned(x, e) || misaligned(residual, e) || misaligned(y, e)) return EMB_ERR_INVALID_ARG;
  const emb::DropoutArgs a{x, ldx, residual, ldr, T, D, mask, y, ldy, dtype == EMB_BF16};
  return launch_status(emb::launch_dropout(a, static_cast<hipStream_t>(stream)));
}

int emb_block_norm(const emb_block_norm_args* a, void* stream) {
  emb::DropMask mask;
  if (a == nullptr || bad_row_dims(a->T, a->D) || bad_dtype(a->stream_dtype) || bad_dtype(a->dtype) ||
      (a->stream_dtype == EMB_BF16 && a->dtype != EMB_BF16) || a->ldx < 0 || a->ldb < 0 || a->ldh < a->D ||
      a->gate_rows < 0 || !(a->eps >= 0.0) || !std::isfinite(a->eps) || !std::isfinite(a->alpha) ||
      !drop_mask(a->p, a->seed, a->seed_dev, &mask) || (a->pre_stats != nullptr && a->ldy < a->D))
    return EMB_ERR_INVALID_ARG;
  if (a->T == 0) return EMB_OK;
  const size_t es = elem_bytes(a->stream_dtype), eb = elem_bytes(a->dtype);
  if (!a->x || !a->branch || !a->h || (a->pre_stats != nullptr && !a->y) || misaligned(a->x, es) ||
      misaligned(a->h, es) || misaligned(a->branch, eb) || misaligned(a->y, eb) || bad_f32(a->gate) ||
      bad_f32(a->post_weight) || bad_f32(a->post_bias) || bad_f32(a->pre_weight) || bad_f32(a->pre_bias) ||
      bad_f32(a->post_stats) || bad_f32(a->pre_stats))
    return EMB_ERR_INVALID_ARG;
  emb_block_norm_args args = *a;
  if (args.gate_rows > args.T) args.gate_rows = args.T;  // one gate; the kernels divide in 32 bits
  return launch_status(emb::launch_block_norm(emb::BlockArgs{&args, mask}, static_cast<hipStream_t>(stream)));
}

size_t emb_block_norm_backward_workspace_bytes(int32_t T, int32_t D, int64_t gate_rows) {
  return bad_row_dims(T, D) || gate_rows < 0 ? 0 : emb::block_norm_grad_workspace_bytes(T, D, gate_rows);
}

int emb_block_norm_backward(const emb_block_norm_grad_args* a, void* stream) {
  emb::DropMask mask;
  if (a == nullptr || bad_row_dims(a->T, a->D) || bad_dtype(a->stream_dtype) || bad_dtype(a->dtype) ||
      (a->stream_dtype == EMB_BF16 && a->dtype != EMB_BF16) || (a->dh != nullptr && a->lddh < 0) ||
      (a->pre_stats != nullptr && a->lddy < 0) || a->ldh < 0 || a->ldb < 0 || a->gate_rows < 0 ||
      !std::isfinite(a->alpha) || !drop_mask(a->p, a->seed, a->seed_dev, &mask) ||
      (a->dx != nullptr && a->lddx < a->D) || (a->dbranch != nullptr && a->lddb < a->D))
    return EMB_ERR_INVALID_ARG;
  if (!a->dx && !a->dbranch && !a->dgate && !a->dpost_weight && !a->dpost_bias && !a->dpre_weight && !a->dpre_bias)
    return EMB_ERR_INVALID_ARG;
  if (bad_f32(a->dgate) || bad_f32(a->dpost_weight) || bad_f32(a->dpost_bias) || bad_f32(a->dpre_weight) ||
      bad_f32(a->dpre_bias) || bad_f32(a->gate) || bad_f32(a->post_weight) || bad_f32(a->post_bias) ||
      bad_f32(a->pre_weight) || bad_f32(a->post_stats) || bad_f32(a->pre_stats))
    return EMB_ERR_INVALID_ARG;
  if (a->T > 0) {
    const size_t es = elem_bytes(a->stream_dtype), eb = elem_bytes(a->dtype);
    if ((a->post_stats == nullptr && (a->dpost_weight != nullptr || a->dpost_bias != nullptr)) ||
        (a->pre_stats == nullptr && (a->dpre_weight != nullptr || a->dpre_bias != nullptr)))
      return EMB_ERR_INVALID_ARG;
    if (!a->branch || (a->pre_stats != nullptr && (!a->dy || !a->h)) || misaligned(a->dh, es) ||
        misaligned(a->h, es) || misaligned(a->dx, es) || misaligned(a->dy, eb) || misaligned(a->branch, eb) ||
        misaligned(a->dbranch, eb))
      return EMB_ERR_INVALID_ARG;
    if (!a->workspace || misaligned(a->workspace, 256)) return EMB_ERR_INVALID_ARG;
    if (a->workspace_bytes < emb::block_norm_grad_workspace_bytes(a->T, a->D, a->gate_rows)) return EMB_ERR_WORKSPACE;
  }
  emb_block_norm_grad_args args = *a;
  if (args.gate_rows > args.T) args.gate_rows = args.T > 0 ? args.T : 1;  // no rows: no gates either
  return launch_status(emb::launch_block_norm_grad(emb::BlockGradArgs{&args, mask}, static_cast<hipStream_t>(stream)));
}

namespace {
constexpr int32_t kMaxTokens = 1 << 22;
bool bad_loss_dims(int32_t T, int64_t V, int32_t D, int32_t dtype) {
  return T < 0 || T > kMaxTokens || V < 1 || V > kMaxV || D < 1 || D > (1 << 16) || bad_dtype(dtype);
}
bool bad_smoothing(double e) { return !(e >= 0.0 && e < 1.0); }
}  // namespace

size_t emb_vocab_loss_workspace_bytes(int32_t T, int64_t V, int32_t D, int32_t dtype) {
  return bad_loss_dims(T, V, D, dtype) ? 0 : emb::loss_workspace_bytes(T, V, D, dtype == EMB_BF16);
}

int emb_vocab_loss(const void* x, int32_t dtype, int64_t ldx, const void* table, int64_t ldw, int32_t T, int64_t V,
                   int32_t D, const int32_t* targets, double smoothing, float* loss, float* lse, void* workspace,
                   size_t workspace_bytes, int32_t* dev_status, void* stream) {
  if (bad_loss_dims(T, V, D, dtype) || bad_smoothing(smoothing) || ldx < 0 || ldw < 0) return EMB_ERR_INVALID_ARG;
  if (T == 0) return EMB_OK;
  if (!x || !table || !targets || !loss || !lse || misaligned(x, elem_bytes(dtype)) ||
      misaligned(table, elem_bytes(dtype)) || bad_f32(targets) || bad_f32(loss) || bad_f32(lse) || !workspace ||
      misaligned(workspace, 256))
    return EMB_ERR_INVALID_ARG;
  const bool is_bf16 = dtype == EMB_BF16;
  if (workspace_bytes < emb::loss_workspace_bytes(T, V, D, is_bf16)) return EMB_ERR_WORKSPACE;
  const emb::LossArgs a{x, ldx, table, ldw, T, V, D, targets, static_cast<float>(smoothing), loss, lse, workspace,
                        dev_status, is_bf16};
  return launch_status(emb::launch_loss(a, static_cast<hipStream_t>(stream)));
}

size_t emb_vocab_loss_backward_workspace_bytes(int32_t T, int64_t V, int32_t D, int32_t dtype) {
  return bad_loss_dims(T, V, D, dtype) ? 0 : emb::loss_grad_workspace_bytes(T, V, D, dtype == EMB_BF16);
}

int emb_vocab_loss_backward(const float* dloss, int32_t dloss_step, const void* x, int32_t dtype, int64_t ldx,
                            const void* table, int64_t ldw, int32_t T, int64_t V, int32_t D, const int32_t* targets,
                            double smoothing, const float* lse, void* dx, int64_t lddx, void* dtable, int64_t lddt,
                            void* workspace, size_t workspace_bytes, int32_t* dev_status, void* stream) {
  if (bad_loss_dims(T, V, D, dtype) || bad_smoothing(smoothing) || ldx < 0 || ldw < 0 ||
      (dloss_step != 0 && dloss_step != 1) || (dx == nullptr && dtable == nullptr) || (dx != nullptr && lddx < D) ||
      (dtable != nullptr && lddt < D))
    return EMB_ERR_INVALID_ARG;
  const size_t e = elem_bytes(dtype);
  if (misaligned(dx, e) || misaligned(dtable, e) || !table || misaligned(table, e) || !workspace ||
      misaligned(workspace, 256))
    return EMB_ERR_INVALID_ARG;
  if (T > 0 && (!dloss || !x || !targets || !lse || misaligned(x, e) || bad_f32(dloss) || bad_f32(targets) || bad_f32(lse)))
    return EMB_ERR_INVALID_ARG;
  const bool is_bf16 = dtype == EMB_BF16;
  if (workspace_bytes < emb::loss_grad_workspace_bytes(T, V, D, is_bf16)) return EMB_ERR_WORKSPACE;
  const emb::LossGradArgs a{dloss, dloss_step, x, ldx, table, ldw, T, V, D, targets, static_cast<float>(smoothing), lse,
                            dx, lddx, dtable, lddt, workspace, dev_status, is_bf16};
  return launch_status(emb::launch_loss_grad(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
