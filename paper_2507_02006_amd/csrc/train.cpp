// Entry points of the training operators: argument checks, then the
// launchers of train.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "arguments.h"
#include "train.h"

using namespace aires;

namespace {

constexpr int64_t kMaxSize = int64_t(1) << 31;

aires_status check_norm_size(int64_t m, int64_t n) {
  if (m < 0 || n < 0) return fail(AIRES_E_DIM, "%lld rows of %lld columns", (long long)m, (long long)n);
  // (column numbers are 32 bits wide, and stepped on past the last)
  if (m > (int64_t(1) << 40) || n > (int64_t(1) << 30))
    return fail(AIRES_E_UNSUPPORTED, "%lld rows of %lld columns", (long long)m, (long long)n);
  return AIRES_OK;
}

aires_status check_xent_size(int64_t t, int64_t d, int64_t v) {
  if (t < 0 || d < 0 || v < 0 || (t > 0 && (d == 0 || v == 0)))
    return fail(AIRES_E_DIM, "%lld rows, %lld features, %lld classes", (long long)t, (long long)d, (long long)v);
  // a stage's offsets are 32 bits wide, a launch has fewer than 2^32 threads
  // (tiles of 128 x 128 of a gradient are 2^23 at most)
  const int64_t outs = ((std::max(t, v) + 127) / 128) * ((d + 127) / 128);
  if (t > (int64_t(1) << 29) || v >= kMaxSize || d >= (int64_t(1) << 21) || outs > (int64_t(1) << 23))
    return fail(AIRES_E_UNSUPPORTED, "%lld rows, %lld features, %lld classes", (long long)t, (long long)d,
                (long long)v);
  return AIRES_OK;
}

}  // namespace

extern "C" {

aires_status aires_layer_norm(const aires_dense* X, const void* gamma, const void* beta, int32_t w_dtype, double eps,
                              const aires_dense* Y, float* mean, float* rstd, void* stream) {
  ST_TRY(check_dense(X, "X"));
  ST_TRY(check_dense(Y, "Y"));
  ST_TRY(check_same(X, "X", Y, "Y"));
  ST_TRY(check_norm_size(X->nrows, X->ncols));
  if (!type_ok(w_dtype)) return fail(AIRES_E_INVALID_ARG, "w_dtype %d invalid", (int)w_dtype);
  if (!std::isfinite(eps) || eps < 0) return fail(AIRES_E_INVALID_ARG, "eps %g invalid", eps);
  if (!mean != !rstd) return fail(AIRES_E_INVALID_ARG, "mean and rstd are wanted together");
  HIP_TRY(kern::layer_norm(mat(X), gamma, beta, w_dtype, (float)eps, mat(Y), mean, rstd, (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_layer_norm_workspace(int64_t m, int64_t n, int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  ST_TRY(check_norm_size(m, n));
  *bytes = kern::layer_norm_workspace(m, n);
  return AIRES_OK;
}

aires_status aires_layer_norm_backward(const aires_dense* dY, const aires_dense* X, const float* mean,
                                       const float* rstd, const void* gamma, int32_t w_dtype, const aires_dense* dX,
                                       void* dgamma, void* dbeta, void* workspace, int64_t workspace_bytes,
                                       void* stream) {
  ST_TRY(check_dense(dY, "dY"));
  ST_TRY(check_dense(X, "X"));
  ST_TRY(check_same(X, "X", dY, "dY"));
  if (dX) {
    ST_TRY(check_dense(dX, "dX"));
    ST_TRY(check_same(X, "X", dX, "dX"));
  }
  ST_TRY(check_norm_size(X->nrows, X->ncols));
  if (!type_ok(w_dtype)) return fail(AIRES_E_INVALID_ARG, "w_dtype %d invalid", (int)w_dtype);
  if (X->nrows > 0 && (!mean || !rstd)) return fail(AIRES_E_INVALID_ARG, "mean or rstd is NULL");
  const int64_t need = dgamma || dbeta ? kern::layer_norm_workspace(X->nrows, X->ncols) : 0;
  if (need > 0 && !workspace) return fail(AIRES_E_INVALID_ARG, "workspace is NULL");
  if (need > 0 && (reinterpret_cast<uintptr_t>(workspace) & 15))
    return fail(AIRES_E_INVALID_ARG, "workspace is not 16-byte aligned");
  if (workspace_bytes < need)
    return fail(AIRES_E_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
  HIP_TRY(kern::layer_norm_backward(mat(dY), mat(X), mean, rstd, gamma, w_dtype, mat(dX), dgamma, dbeta,
                                    (float*)workspace, (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_linear_xent_workspace(int64_t t, int64_t d, int64_t v, int32_t dtype, int32_t grads,
                                         int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  if (!type_ok(dtype)) return fail(AIRES_E_INVALID_ARG, "dtype %d invalid", (int)dtype);
  ST_TRY(check_xent_size(t, d, v));
  *bytes = kern::linear_xent_workspace(t, d, v, dtype, grads != 0);
  return AIRES_OK;
}

aires_status aires_linear_xent(const aires_dense* H, const aires_dense* W, const void* labels, int32_t labels_i64,
                               int32_t reduction, double grad_scale, float* loss, float* row_loss,
                               const aires_dense* dH, const aires_dense* dW, void* workspace,
                               int64_t workspace_bytes, void* stream) {
  ST_TRY(check_dense(H, "H"));
  ST_TRY(check_dense(W, "W"));
  if (H->ncols != W->ncols || H->dtype != W->dtype)
    return fail(AIRES_E_DIM, "H has %lld columns of type %d, W %lld of type %d", (long long)H->ncols, (int)H->dtype,
                (long long)W->ncols, (int)W->dtype);
  ST_TRY(check_xent_size(H->nrows, H->ncols, W->nrows));
  if (!dH != !dW) return fail(AIRES_E_INVALID_ARG, "dH and dW are wanted together");
  if (dH) {
    ST_TRY(check_dense(dH, "dH"));
    ST_TRY(check_same(H, "H", dH, "dH"));
    ST_TRY(check_dense(dW, "dW"));
    ST_TRY(check_same(W, "W", dW, "dW"));
    if (dH->dtype != H->dtype || dW->dtype != W->dtype)
      return fail(AIRES_E_DIM, "dH and dW have H's and W's type");
  }
  if (reduction != AIRES_REDUCE_MEAN && reduction != AIRES_REDUCE_SUM)
    return fail(AIRES_E_INVALID_ARG, "reduction %d invalid", (int)reduction);
  if (!std::isfinite(grad_scale)) return fail(AIRES_E_INVALID_ARG, "grad_scale is not finite");
  if (!loss || (H->nrows > 0 && !labels)) return fail(AIRES_E_INVALID_ARG, "loss or labels is NULL");
  const int64_t need = kern::linear_xent_workspace(H->nrows, H->ncols, W->nrows, H->dtype, dH != nullptr);
  if (need > 0 && !workspace) return fail(AIRES_E_INVALID_ARG, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 15)
    return fail(AIRES_E_INVALID_ARG, "workspace is not 16-byte aligned");
  if (workspace_bytes < need)
    return fail(AIRES_E_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
  kern::XentArgs x{mat(H), mat(W), mat(dH), mat(dW), labels, labels_i64, reduction == AIRES_REDUCE_MEAN,
                   (float)grad_scale, loss, row_loss, workspace};
  HIP_TRY(kern::linear_xent(x, (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_adamw(const aires_adamw_tensor* tensors, int64_t count, const aires_adamw_opts* opts,
                         void* stream) {
  return aires_adamw_scaled(tensors, count, opts, nullptr, stream);
}

aires_status aires_adamw_scaled(const aires_adamw_tensor* tensors, int64_t count, const aires_adamw_opts* opts,
                                const float* grad_scale, void* stream) {
  if (!opts || opts->struct_size != sizeof(aires_adamw_opts)) return fail(AIRES_E_INVALID_ARG, "bad options");
  if (count < 0 || (count > 0 && !tensors)) return fail(AIRES_E_INVALID_ARG, "%lld tensors", (long long)count);
  const aires_adamw_opts& o = *opts;
  if (o.step < 1) return fail(AIRES_E_INVALID_ARG, "step %lld: steps count from 1", (long long)o.step);
  for (double b : {o.beta1, o.beta2})
    if (!(b >= 0.0 && b < 1.0)) return fail(AIRES_E_INVALID_ARG, "beta %g outside [0, 1)", b);
  if (!std::isfinite(o.lr) || !std::isfinite(o.weight_decay) || !std::isfinite(o.grad_scale) || !std::isfinite(o.eps) ||
      o.eps < 0)
    return fail(AIRES_E_INVALID_ARG, "lr, weight_decay, grad_scale or eps invalid");
  std::vector<kern::AdamWTensor> list;
  try {
    list.reserve((size_t)count);
  } catch (const std::exception&) {
    return fail(AIRES_E_OOM, "no host memory for %lld descriptors", (long long)count);
  }
  for (int64_t k = 0; k < count; ++k) {
    const aires_adamw_tensor& t = tensors[k];
    const long long at = (long long)k;
    if (t.n < 0) return fail(AIRES_E_DIM, "tensor %lld has %lld values", at, (long long)t.n);
    if (!type_ok(t.param_dtype) || !type_ok(t.grad_dtype) || (t.copy && !type_ok(t.copy_dtype)))
      return fail(AIRES_E_INVALID_ARG, "tensor %lld: invalid type", at);
    if (t.n == 0) continue;
    if (t.n > (int64_t(1) << 35)) return fail(AIRES_E_UNSUPPORTED, "tensor %lld has %lld values", at, (long long)t.n);
    if (!t.param || !t.grad || !t.exp_avg || !t.exp_avg_sq)
      return fail(AIRES_E_INVALID_ARG, "tensor %lld: NULL array", at);
    if (!t.exp_avg_scale != !t.exp_avg_sq_scale)
      return fail(AIRES_E_INVALID_ARG, "tensor %lld: both moments are held in 8 bits, or none", at);
    list.push_back(kern::AdamWTensor{t.param, t.grad, t.exp_avg, t.exp_avg_sq, t.exp_avg_scale, t.exp_avg_sq_scale,
                                     t.copy, t.n, kern::adamw_seed(o.seed, k), (uint8_t)t.param_dtype,
                                     (uint8_t)t.grad_dtype, (uint8_t)t.copy_dtype});
  }
  kern::AdamWStep s;
  s.beta1 = (float)o.beta1;
  s.one_beta1 = (float)(1.0 - o.beta1);
  s.beta2 = (float)o.beta2;
  s.one_beta2 = (float)(1.0 - o.beta2);
  s.eps = (float)o.eps;
  s.decay = (float)(1.0 - o.lr * o.weight_decay);
  s.rate = (float)(o.lr / (1.0 - std::pow(o.beta1, (double)o.step)));
  s.inv_root = (float)(1.0 / std::sqrt(1.0 - std::pow(o.beta2, (double)o.step)));
  s.grad_scale = (float)o.grad_scale;
  HIP_TRY(kern::adamw(list.data(), (int64_t)list.size(), s, grad_scale, (hipStream_t)stream));
  return AIRES_OK;
}

}  // extern "C"
