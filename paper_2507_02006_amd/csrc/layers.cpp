// Entry points of the operators of layers: argument checks, then the launchers
// of layers.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <vector>

#include "arguments.h"
#include "layers.h"

using namespace aires;

namespace {

constexpr int64_t kMostCols = int64_t(1) << 30;

aires_status check_rows(int64_t m, int64_t n) {
  if (m < 0 || n < 0) return fail(AIRES_E_DIM, "%lld rows of %lld columns", (long long)m, (long long)n);
  // (column numbers are 32 bits wide, and stepped on past the last)
  if (m > (int64_t(1) << 40) || n > kMostCols)
    return fail(AIRES_E_UNSUPPORTED, "%lld rows of %lld columns", (long long)m, (long long)n);
  return AIRES_OK;
}

aires_status check_held(const aires_dense8* q, const char* name) {
  if (!q) return fail(AIRES_E_INVALID_ARG, "%s is NULL", name);
  if (q->nrows < 0 || q->ncols < 0)
    return fail(AIRES_E_DIM, "%s is %lld x %lld", name, (long long)q->nrows, (long long)q->ncols);
  if (q->tile != 1 && q->tile != AIRES_BLOCK8) return fail(AIRES_E_INVALID_ARG, "%s: tile %d", name, (int)q->tile);
  if (q->nrows > 0 && q->ncols > 0) {
    if (!q->codes || !q->scales) return fail(AIRES_E_INVALID_ARG, "%s has no codes or no scales", name);
    if (q->ld < q->ncols || q->ld_scales < (q->ncols + AIRES_BLOCK8 - 1) / AIRES_BLOCK8)
      return fail(AIRES_E_INVALID_ARG, "%s: strides %lld and %lld for %lld columns", name, (long long)q->ld,
                  (long long)q->ld_scales, (long long)q->ncols);
    if (reinterpret_cast<uintptr_t>(q->scales) % 4) return fail(AIRES_E_INVALID_ARG, "%s: scales are not aligned", name);
  }
  return AIRES_OK;
}

kern::Held held(const aires_dense8* q) {
  if (!q) return kern::Held{nullptr, nullptr, 0, 0, 0, 0, 1};
  return kern::Held{q->codes, q->scales, q->nrows, q->ncols, q->ld, q->ld_scales, q->tile};
}

// An output in an input's place lies there exactly.
aires_status check_place(const aires_dense* out, const char* on, const aires_dense* in, const char* in_name) {
  if (!out || !in || out->data != in->data || out->nrows == 0 || out->ncols == 0) return AIRES_OK;
  if (out->dtype != in->dtype || (out->nrows > 1 && out->ld != in->ld))
    return fail(AIRES_E_INVALID_ARG, "%s lies where %s does, in another type or stride", on, in_name);
  return AIRES_OK;
}

aires_status check_workspace(const void* ws, int64_t have, int64_t need) {
  if (need > 0 && !ws) return fail(AIRES_E_INVALID_ARG, "workspace is NULL");
  if (need > 0 && (reinterpret_cast<uintptr_t>(ws) & 15))
    return fail(AIRES_E_INVALID_ARG, "workspace is not 16-byte aligned");
  if (have < need)
    return fail(AIRES_E_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)have, (long long)need);
  return AIRES_OK;
}

aires_status check_product(int64_t m, int64_t n, int64_t k) {
  if (m < 0 || n < 0 || k < 0)
    return fail(AIRES_E_DIM, "product of %lld x %lld x %lld", (long long)m, (long long)n, (long long)k);
  // (a launch has fewer than 2^32 threads: 512 for 16 columns of Y, or 256 for a tile)
  if (m > (int64_t(1) << 26) || n > (int64_t(1) << 26) || k > (int64_t(1) << 23) ||
      ((m + 127) / 128) * ((n + 127) / 128) > (int64_t(1) << 22))
    return fail(AIRES_E_UNSUPPORTED, "product of %lld x %lld x %lld", (long long)m, (long long)n, (long long)k);
  return AIRES_OK;
}

aires_status check_operands(const aires_dense8* A, const aires_dense8* B) {
  ST_TRY(check_held(A, "A"));
  ST_TRY(check_held(B, "B"));
  if (A->ncols != B->ncols)
    return fail(AIRES_E_DIM, "A has %lld columns, B %lld", (long long)A->ncols, (long long)B->ncols);
  ST_TRY(check_product(A->nrows, B->nrows, A->ncols));
  if (A->tile != 1) return fail(AIRES_E_INVALID_ARG, "A has scales for each row (tile 1)");
  // (offsets within a tile are 32 bits wide)
  if (A->ncols > 0)
    for (const aires_dense8* q : {A, B})
      if (q->nrows > 1 && (q->ld > (int64_t(1) << 23) || q->ld_scales > (int64_t(1) << 21)))
        return fail(AIRES_E_UNSUPPORTED, "strides of %lld and %lld", (long long)q->ld, (long long)q->ld_scales);
  return AIRES_OK;
}

aires_status check_scores(int64_t t, int64_t v, int32_t top) {
  if (t < 0 || v < 0 || (t > 0 && v == 0))
    return fail(AIRES_E_DIM, "%lld rows of %lld scores", (long long)t, (long long)v);
  if (top < 0 || top > AIRES_MAX_TOP) return fail(AIRES_E_INVALID_ARG, "top %d outside [0, %d]", (int)top, AIRES_MAX_TOP);
  if (t > 0 && top > v) return fail(AIRES_E_DIM, "%d alternatives of %lld classes", (int)top, (long long)v);
  if (t > (int64_t(1) << 40) || v >= kMostCols)
    return fail(AIRES_E_UNSUPPORTED, "%lld rows of %lld scores", (long long)t, (long long)v);
  return AIRES_OK;
}

aires_status check_count(int64_t count) {
  if (count < 0) return fail(AIRES_E_INVALID_ARG, "%lld tensors", (long long)count);
  if (count > (int64_t(1) << 24)) return fail(AIRES_E_UNSUPPORTED, "%lld tensors", (long long)count);
  return AIRES_OK;
}

// Clipped gradients lie in memory of their own: no two of them overlap, and none
// overlaps a gradient but, exactly, its own.
aires_status check_outs(const std::vector<kern::GradTensor>& list) {
  struct Span {
    uintptr_t begin, end;
    size_t k;
  };
  const auto of = [](const void* p, int64_t n, int type) {
    const uintptr_t b = reinterpret_cast<uintptr_t>(p);
    return Span{b, b + (uintptr_t)n * (type == AIRES_F32 ? 4 : 2), 0};
  };
  std::vector<Span> outs(list.size());
  for (size_t k = 0; k < list.size(); ++k) {
    outs[k] = of(list[k].out, list[k].n, list[k].ot);
    outs[k].k = k;
  }
  std::sort(outs.begin(), outs.end(), [](const Span& a, const Span& b) { return a.begin < b.begin; });
  for (size_t i = 0; i + 1 < outs.size(); ++i)
    if (outs[i + 1].begin < outs[i].end) return fail(AIRES_E_INVALID_ARG, "clipped gradients overlap each other");
  for (size_t k = 0; k < list.size(); ++k) {
    const Span g = of(list[k].g, list[k].n, list[k].gt);
    auto o = std::upper_bound(outs.begin(), outs.end(), g.begin, [](uintptr_t b, const Span& x) { return b < x.end; });
    for (; o != outs.end() && o->begin < g.end; ++o)
      if (o->k != k || list[k].out != list[k].g)
        return fail(AIRES_E_INVALID_ARG, "a clipped gradient overlaps another gradient");
  }
  return AIRES_OK;
}

aires_status grad_norm(const aires_grad_tensor* tensors, int64_t count, double max_norm, float* norm, float* scale,
                       bool clip, void* workspace, int64_t workspace_bytes, void* stream) {
  ST_TRY(check_count(count));
  if (count > 0 && !tensors) return fail(AIRES_E_INVALID_ARG, "tensors is NULL");
  if (!(max_norm >= 0)) return fail(AIRES_E_INVALID_ARG, "max_norm %g", max_norm);
  if (!norm) return fail(AIRES_E_INVALID_ARG, "norm is NULL");
  std::vector<kern::GradTensor> list;
  try {
    list.reserve((size_t)count);
  } catch (const std::exception&) {
    return fail(AIRES_E_OOM, "no host memory for %lld descriptors", (long long)count);
  }
  for (int64_t k = 0; k < count; ++k) {
    const aires_grad_tensor& t = tensors[k];
    const long long at = (long long)k;
    if (t.n < 0) return fail(AIRES_E_DIM, "tensor %lld has %lld values", at, (long long)t.n);
    if (!type_ok(t.grad_dtype) || (clip && !type_ok(t.out_dtype)))
      return fail(AIRES_E_INVALID_ARG, "tensor %lld: invalid type", at);
    if (t.n == 0) continue;
    if (t.n > (int64_t(1) << 35)) return fail(AIRES_E_UNSUPPORTED, "tensor %lld has %lld values", at, (long long)t.n);
    if (!t.grad || (clip && !t.out)) return fail(AIRES_E_INVALID_ARG, "tensor %lld: NULL array", at);
    if (clip && t.out == t.grad && t.out_dtype != t.grad_dtype)
      return fail(AIRES_E_INVALID_ARG, "tensor %lld: out lies where grad does, in another type", at);
    list.push_back(kern::GradTensor{t.grad, t.out, t.n, (uint8_t)t.grad_dtype, (uint8_t)t.out_dtype});
  }
  if (clip) {
    try {
      ST_TRY(check_outs(list));
    } catch (const std::exception&) {
      return fail(AIRES_E_OOM, "no host memory for %lld descriptors", (long long)count);
    }
  }
  ST_TRY(check_workspace(workspace, workspace_bytes, kern::grad_norm_workspace(count)));
  HIP_TRY(kern::grad_norm(list.data(), (int64_t)list.size(), max_norm, norm, scale, clip, workspace,
                          (hipStream_t)stream));
  return AIRES_OK;
}

}  // namespace

extern "C" {

aires_status aires_grad_norm_workspace(int64_t count, int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  ST_TRY(check_count(count));
  *bytes = kern::grad_norm_workspace(count);
  return AIRES_OK;
}

aires_status aires_grad_norm(const aires_grad_tensor* tensors, int64_t count, double max_norm, float* norm,
                             float* scale, void* workspace, int64_t workspace_bytes, void* stream) {
  return grad_norm(tensors, count, max_norm, norm, scale, false, workspace, workspace_bytes, stream);
}

aires_status aires_clip_grads(const aires_grad_tensor* tensors, int64_t count, double max_norm, float* norm,
                              void* workspace, int64_t workspace_bytes, void* stream) {
  return grad_norm(tensors, count, max_norm, norm, nullptr, true, workspace, workspace_bytes, stream);
}

aires_status aires_quantize8(const aires_dense* X, const aires_dense8* Q, const aires_dense8* Qt, void* stream) {
  ST_TRY(check_dense(X, "X"));
  if (!Q && !Qt) return fail(AIRES_E_INVALID_ARG, "neither Q nor Qt is given");
  if (X->nrows > kMostCols || X->ncols > kMostCols)
    return fail(AIRES_E_UNSUPPORTED, "%lld x %lld", (long long)X->nrows, (long long)X->ncols);
  if (Q) {
    ST_TRY(check_held(Q, "Q"));
    if (Q->nrows != X->nrows || Q->ncols != X->ncols) return fail(AIRES_E_DIM, "X and Q differ in size");
  }
  if (Qt) {
    ST_TRY(check_held(Qt, "Qt"));
    if (Qt->nrows != X->ncols || Qt->ncols != X->nrows) return fail(AIRES_E_DIM, "X and Qt transposed differ in size");
  }
  if (Q && Qt && Q->tile != Qt->tile) return fail(AIRES_E_INVALID_ARG, "Q and Qt have different tiles");
  HIP_TRY(kern::quantize8(mat(X), held(Q), held(Qt), (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_matmul8_workspace(const aires_dense8* A, const aires_dense8* B, int32_t dtype, int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  ST_TRY(check_operands(A, B));
  if (!type_ok(dtype)) return fail(AIRES_E_INVALID_ARG, "dtype %d invalid", (int)dtype);
  *bytes = kern::matmul8_workspace(held(A), held(B), dtype);
  return AIRES_OK;
}

aires_status aires_matmul8(const aires_dense8* A, const aires_dense8* B, const aires_dense* Y, void* workspace,
                           int64_t workspace_bytes, void* stream) {
  ST_TRY(check_operands(A, B));
  ST_TRY(check_dense(Y, "Y"));
  if (Y->nrows != A->nrows || Y->ncols != B->nrows)
    return fail(AIRES_E_DIM, "A has %lld rows, B %lld, Y is %lld x %lld", (long long)A->nrows, (long long)B->nrows,
                (long long)Y->nrows, (long long)Y->ncols);
  ST_TRY(check_workspace(workspace, workspace_bytes, kern::matmul8_workspace(held(A), held(B), Y->dtype)));
  HIP_TRY(kern::matmul8(held(A), held(B), mat(Y), workspace, (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_rms_norm(const aires_dense* X, const aires_dense* R, const void* gamma, int32_t w_dtype, double eps,
                            const aires_dense* S, const aires_dense* Y, const aires_dense8* Y8, float* rstd,
                            void* stream) {
  ST_TRY(check_dense(X, "X"));
  if (!R != !S) return fail(AIRES_E_INVALID_ARG, "R and S go together");
  if (!Y == !Y8) return fail(AIRES_E_INVALID_ARG, "one of Y and Y8 is wanted");
  if (R) {
    ST_TRY(check_dense(R, "R"));
    ST_TRY(check_dense(S, "S"));
    ST_TRY(check_same(X, "X", R, "R"));
    ST_TRY(check_same(X, "X", S, "S"));
    ST_TRY(check_place(S, "S", X, "X"));
    ST_TRY(check_place(S, "S", R, "R"));
  }
  if (Y) {
    ST_TRY(check_dense(Y, "Y"));
    ST_TRY(check_same(X, "X", Y, "Y"));
  } else {
    ST_TRY(check_held(Y8, "Y8"));
    if (Y8->nrows != X->nrows || Y8->ncols != X->ncols) return fail(AIRES_E_DIM, "X and Y8 differ in size");
    if (Y8->tile != 1) return fail(AIRES_E_INVALID_ARG, "Y8 has scales for each row (tile 1)");
  }
  ST_TRY(check_rows(X->nrows, X->ncols));
  if (!type_ok(w_dtype)) return fail(AIRES_E_INVALID_ARG, "w_dtype %d invalid", (int)w_dtype);
  if (!std::isfinite(eps) || eps < 0) return fail(AIRES_E_INVALID_ARG, "eps %g invalid", eps);
  HIP_TRY(kern::rms_norm(mat(X), mat(R), gamma, w_dtype, (float)eps, mat(S), mat(Y), held(Y8), rstd,
                         (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_rms_norm_workspace(int64_t m, int64_t n, int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  ST_TRY(check_rows(m, n));
  *bytes = kern::rms_norm_workspace(m, n);
  return AIRES_OK;
}

aires_status aires_rms_norm_backward(const aires_dense* dY, const aires_dense* S, const float* rstd,
                                     const void* gamma, int32_t w_dtype, const aires_dense* dS,
                                     const aires_dense* dX, void* dgamma, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
  ST_TRY(check_dense(dY, "dY"));
  ST_TRY(check_dense(S, "S"));
  ST_TRY(check_same(S, "S", dY, "dY"));
  if (dS) {
    ST_TRY(check_dense(dS, "dS"));
    ST_TRY(check_same(S, "S", dS, "dS"));
  }
  if (dX) {
    ST_TRY(check_dense(dX, "dX"));
    ST_TRY(check_same(S, "S", dX, "dX"));
    ST_TRY(check_place(dX, "dX", dS, "dS"));
  }
  ST_TRY(check_rows(S->nrows, S->ncols));
  if (!type_ok(w_dtype)) return fail(AIRES_E_INVALID_ARG, "w_dtype %d invalid", (int)w_dtype);
  if (S->nrows > 0 && !rstd) return fail(AIRES_E_INVALID_ARG, "rstd is NULL");
  ST_TRY(check_workspace(workspace, workspace_bytes, dgamma ? kern::rms_norm_workspace(S->nrows, S->ncols) : 0));
  HIP_TRY(kern::rms_norm_backward(mat(dY), mat(S), rstd, gamma, w_dtype, mat(dS), mat(dX), dgamma, (float*)workspace,
                                  (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_log_probs_workspace(int64_t t, int64_t v, int32_t top, int64_t* bytes) {
  if (!bytes) return fail(AIRES_E_INVALID_ARG, "bytes is NULL");
  ST_TRY(check_scores(t, v, top));
  *bytes = kern::log_probs_workspace(t, v, top);
  return AIRES_OK;
}

aires_status aires_log_probs(const aires_dense* Z, const void* labels, int32_t labels_i64, int32_t top, float* logp,
                             float* entropy, float* lse, float* top_logp, int64_t* top_index, void* workspace,
                             int64_t workspace_bytes, void* stream) {
  return aires_log_probs_rest(Z, labels, labels_i64, top, logp, entropy, lse, nullptr, top_logp, top_index, workspace,
                              workspace_bytes, stream);
}

aires_status aires_log_probs_rest(const aires_dense* Z, const void* labels, int32_t labels_i64, int32_t top,
                                  float* logp, float* entropy, float* lse, float* lse_rest, float* top_logp,
                                  int64_t* top_index, void* workspace, int64_t workspace_bytes, void* stream) {
  ST_TRY(check_dense(Z, "Z"));
  ST_TRY(check_scores(Z->nrows, Z->ncols, top));
  if (Z->nrows > 0) {
    if (!labels != !logp) return fail(AIRES_E_INVALID_ARG, "labels and logp go together");
    if (top > 0 && (!top_logp || !top_index)) return fail(AIRES_E_INVALID_ARG, "top_logp or top_index is NULL");
    if (lse_rest && !lse) return fail(AIRES_E_INVALID_ARG, "lse_rest without lse");
  }
  ST_TRY(check_workspace(workspace, workspace_bytes, kern::log_probs_workspace(Z->nrows, Z->ncols, top)));
  const kern::LogProbs a{mat(Z), labels, labels_i64, top, logp, entropy, lse, lse_rest, top_logp, top_index};
  HIP_TRY(kern::log_probs(a, workspace, (hipStream_t)stream));
  return AIRES_OK;
}

aires_status aires_log_probs_backward(const aires_dense* Z, const void* labels, int32_t labels_i64, const float* lse,
                                      const float* entropy, const float* dlogp, const float* dentropy,
                                      const aires_dense* dZ, void* stream) {
  return aires_log_probs_backward_rest(Z, labels, labels_i64, lse, nullptr, entropy, dlogp, dentropy, dZ, stream);
}

aires_status aires_log_probs_backward_rest(const aires_dense* Z, const void* labels, int32_t labels_i64,
                                           const float* lse, const float* lse_rest, const float* entropy,
                                           const float* dlogp, const float* dentropy, const aires_dense* dZ,
                                           void* stream) {
  ST_TRY(check_dense(Z, "Z"));
  ST_TRY(check_dense(dZ, "dZ"));
  ST_TRY(check_same(Z, "Z", dZ, "dZ"));
  ST_TRY(check_place(dZ, "dZ", Z, "Z"));
  ST_TRY(check_scores(Z->nrows, Z->ncols, 0));
  if (Z->nrows > 0 && (!lse || (dentropy && !entropy) || (dlogp && !labels)))
    return fail(AIRES_E_INVALID_ARG, "lse, entropy or labels is NULL");
  HIP_TRY(kern::log_probs_backward(mat(Z), labels, labels_i64, lse, lse_rest, entropy, dlogp, dentropy,
                                   mat(dZ), (hipStream_t)stream));
  return AIRES_OK;
}

}  // extern "C"
