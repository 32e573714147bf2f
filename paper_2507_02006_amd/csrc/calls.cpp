// The training calls of include/aires.h over torch tensors: checks of the
// arguments, outputs and workspaces from torch's allocator, and the call.
// Written in C++ because these calls are often shorter than their checks are
// in Python (a layer norm of 128 rows: 3.5 us on the device, 12 us to issue
// through ctypes; 19 tensors of an AdamW step: 9 and 40).
#include <torch/extension.h>

#include <string>
#include <vector>

#include "../../include/aires.h"

namespace py = pybind11;

namespace {

py::object g_error;  // AiresError(status, where)

void check(aires_status s, const char* where) {
  if (s == AIRES_OK) return;
  py::object e = g_error((int)s, where);
  PyErr_SetObject(g_error.ptr(), e.ptr());
  throw py::error_already_set();
}

[[noreturn]] void bad_value(const std::string& text) { throw py::value_error(text); }

int32_t dtype_of(at::ScalarType t) {
  switch (t) {
    case at::kFloat: return AIRES_F32;
    case at::kBFloat16: return AIRES_BF16;
    case at::kHalf: return AIRES_F16;
    default: throw py::type_error(std::string("expected float32, bfloat16 or float16, got ") + c10::toString(t));
  }
}

aires_dense dense(const at::Tensor& x, const char* name) {
  if (x.dim() != 2 || !x.is_cuda()) bad_value(std::string(name) + " must be a device matrix");
  const int64_t m = x.size(0), n = x.size(1), ld = m > 1 ? x.stride(0) : n;
  if ((n > 1 && m > 0 && x.stride(1) != 1) || (m > 1 && n > 0 && ld < n))
    bad_value(std::string(name) + " needs unit column stride and rows that do not overlap");
  return aires_dense{m, n, ld, dtype_of(x.scalar_type()), 0, x.data_ptr()};
}

void* vector(const at::Tensor& x, int64_t n, const char* name) {
  if (x.dim() != 1 || x.size(0) != n || !x.is_cuda() || !x.is_contiguous())
    bad_value(std::string(name) + " must be a contiguous device vector of " + std::to_string(n) + " values");
  return x.data_ptr();
}

void same_device(const at::Tensor& first, const at::Tensor& x) {
  if (x.device() != first.device())
    bad_value("tensors on " + first.device().str() + " and " + x.device().str());
}

using Maybe = std::optional<at::Tensor>;

// x was written through its address: a backward pass that has kept it is to
// notice.  (Inference tensors count no versions.)
void written(const at::Tensor& x) {
  if (!x.is_inference()) x.unsafeGetTensorImpl()->bump_version();
}

py::object or_none(const at::Tensor& t) { return t.defined() ? py::cast(t) : py::none(); }

py::tuple layer_norm(const at::Tensor& X, const Maybe& gamma, const Maybe& beta, double eps,
                     std::optional<at::ScalarType> out_dtype, bool stats, const Maybe& out, uintptr_t stream) {
  const aires_dense x = dense(X, "X");
  const int64_t m = x.nrows, n = x.ncols;
  if (gamma && beta && gamma->scalar_type() != beta->scalar_type())
    throw py::type_error("gamma and beta have different types");
  const void *g = nullptr, *b = nullptr;
  int32_t wt = AIRES_F32;
  for (const Maybe* w : {&gamma, &beta})
    if (*w) {
      same_device(X, **w);
      wt = dtype_of((*w)->scalar_type());
    }
  if (gamma) g = vector(*gamma, n, "gamma");
  if (beta) b = vector(*beta, n, "beta");
  if (out) same_device(X, *out);
  if (out && out_dtype && out->scalar_type() != *out_dtype) throw py::type_error("out has another type than out_dtype");
  const at::Tensor Y = out ? *out : at::empty({m, n}, X.options().dtype(out_dtype.value_or(X.scalar_type())));
  const aires_dense y = dense(Y, "out");
  at::Tensor mean, rstd;
  if (stats) {
    mean = at::empty({m}, X.options().dtype(at::kFloat));
    rstd = at::empty({m}, X.options().dtype(at::kFloat));
  }
  // (an empty vector has no address: nothing is written then)
  const bool st = stats && m > 0;
  check(aires_layer_norm(&x, g, b, wt, eps, &y, st ? mean.data_ptr<float>() : nullptr,
                         st ? rstd.data_ptr<float>() : nullptr, (void*)stream),
        "aires_layer_norm");
  if (out) written(*out);
  if (!stats) return py::make_tuple(Y, py::none(), py::none());
  return py::make_tuple(Y, mean, rstd);
}

py::tuple layer_norm_backward(const at::Tensor& dY, const at::Tensor& X, const at::Tensor& mean,
                              const at::Tensor& rstd, const Maybe& gamma, bool need_dx, bool need_weights,
                              std::optional<at::ScalarType> dx_dtype, uintptr_t stream) {
  const aires_dense dy = dense(dY, "dY"), x = dense(X, "X");
  const int64_t m = x.nrows, n = x.ncols;
  if (dy.nrows != m || dy.ncols != n) bad_value("dY and X differ in size");
  const void* g = gamma ? vector(*gamma, n, "gamma") : nullptr;
  const void *mu = vector(mean, m, "mean"), *r = vector(rstd, m, "rstd");
  if (mean.scalar_type() != at::kFloat || rstd.scalar_type() != at::kFloat)
    throw py::type_error("mean and rstd must be float32");
  same_device(X, dY);
  same_device(X, mean);
  same_device(X, rstd);
  if (gamma) same_device(X, *gamma);
  const at::ScalarType w = gamma ? gamma->scalar_type() : at::kFloat;
  const int32_t wt = dtype_of(w);
  at::Tensor dX, dg, db, work;
  aires_dense dx{};
  if (need_dx) {
    dX = at::empty({m, n}, X.options().dtype(dx_dtype.value_or(X.scalar_type())));
    dx = dense(dX, "dX");
  }
  int64_t need = 0;
  if (need_weights) {
    check(aires_layer_norm_workspace(m, n, &need), "aires_layer_norm_workspace");
    dg = at::empty({n}, X.options().dtype(w));
    db = at::empty({n}, X.options().dtype(w));
    work = at::empty({need}, X.options().dtype(at::kByte));
  }
  check(aires_layer_norm_backward(&dy, &x, (const float*)mu, (const float*)r, g, wt, need_dx ? &dx : nullptr,
                                  need_weights ? dg.data_ptr() : nullptr, need_weights ? db.data_ptr() : nullptr,
                                  need_weights ? work.data_ptr() : nullptr, need, (void*)stream),
        "aires_layer_norm_backward");
  return py::make_tuple(or_none(dX), or_none(dg), or_none(db));
}

py::tuple linear_xent(const at::Tensor& H, const at::Tensor& W, const at::Tensor& labels, bool mean, bool grads,
                      double grad_scale, uintptr_t stream) {
  if (labels.scalar_type() != at::kInt && labels.scalar_type() != at::kLong)
    throw py::type_error("labels must be int32 or int64");
  const aires_dense h = dense(H, "H"), w = dense(W, "W");
  if (h.ncols != w.ncols || h.dtype != w.dtype) bad_value("H and W differ in columns or type");
  const void* y = vector(labels, h.nrows, "labels");
  same_device(H, W);
  same_device(H, labels);
  int64_t need = 0;
  check(aires_linear_xent_workspace(h.nrows, h.ncols, w.nrows, h.dtype, grads, &need), "aires_linear_xent_workspace");
  const at::Tensor work = at::empty({need}, H.options().dtype(at::kByte));
  const at::Tensor loss = at::empty({}, H.options().dtype(at::kFloat));
  const at::Tensor rows = at::empty({h.nrows}, H.options().dtype(at::kFloat));
  at::Tensor dH, dW;
  aires_dense dh{}, dw{};
  if (grads) {
    dH = at::empty({h.nrows, h.ncols}, H.options());
    dW = at::empty({w.nrows, w.ncols}, W.options());
    dh = dense(dH, "dH");
    dw = dense(dW, "dW");
  }
  check(aires_linear_xent(&h, &w, y, labels.scalar_type() == at::kLong, mean ? AIRES_REDUCE_MEAN : AIRES_REDUCE_SUM,
                          grad_scale, loss.data_ptr<float>(), (float*)rows.data_ptr(), grads ? &dh : nullptr,
                          grads ? &dw : nullptr, work.data_ptr(), need, (void*)stream),
        "aires_linear_xent");
  return py::make_tuple(loss, rows, or_none(dH), or_none(dW));
}

constexpr at::ScalarType kCodes = at::kFloat8_e4m3fn;

int64_t blocks(int64_t n) { return (n + AIRES_BLOCK8 - 1) / AIRES_BLOCK8; }

// A matrix held in 8 bits: a pair of codes and scales.  tile = 0: from the scales' number.
aires_dense8 held(const at::Tensor& codes, const at::Tensor& scales, int32_t tile, const std::string& name) {
  if (codes.dim() != 2 || !codes.is_cuda() || codes.scalar_type() != kCodes)
    bad_value(name + ": codes must be a device matrix of float8_e4m3fn");
  const int64_t m = codes.size(0), n = codes.size(1), ld = m > 1 ? codes.stride(0) : n;
  if ((n > 1 && m > 0 && codes.stride(1) != 1) || (m > 1 && n > 0 && ld < n))
    bad_value(name + ": codes need unit column stride and rows that do not overlap");
  if (scales.dim() != 2 || scales.scalar_type() != at::kFloat || scales.device() != codes.device())
    bad_value(name + ": scales must be a float32 matrix on the codes' device");
  const int64_t rows = scales.size(0), b = blocks(n), lds = rows > 1 ? scales.stride(0) : b;
  if (tile == 0) tile = rows == m ? 1 : AIRES_BLOCK8;
  if (rows != (tile == 1 ? m : blocks(m)) || scales.size(1) != b)
    bad_value(name + ": " + std::to_string(rows) + " x " + std::to_string(scales.size(1)) + " scales for " +
              std::to_string(m) + " x " + std::to_string(n) + " codes");
  if ((b > 1 && rows > 0 && scales.stride(1) != 1) || (rows > 1 && b > 0 && lds < b))
    bad_value(name + ": scales need unit column stride and rows that do not overlap");
  return aires_dense8{m, n, ld, (uint8_t*)codes.data_ptr(), (float*)scales.data_ptr(), lds, tile, 0};
}

const at::Tensor& part(const py::tuple& pair, int i, const char* name) {
  const PyObject* x = PyTuple_GET_SIZE(pair.ptr()) == 2 ? PyTuple_GET_ITEM(pair.ptr(), i) : nullptr;
  if (!x || !THPVariable_Check(const_cast<PyObject*>(x))) bad_value(std::string(name) + " must be a pair of codes and scales");
  return THPVariable_Unpack(const_cast<PyObject*>(x));
}

struct New8 {
  at::Tensor codes, scales;
  aires_dense8 q;
  New8() : q{} {}
  New8(int64_t m, int64_t n, bool tiles, const at::TensorOptions& o)
      : codes(at::empty({m, n}, o.dtype(kCodes))),
        scales(at::empty({tiles ? blocks(m) : m, blocks(n)}, o.dtype(at::kFloat))) {
    q = aires_dense8{m, n, n, (uint8_t*)codes.data_ptr(), (float*)scales.data_ptr(), blocks(n), tiles ? AIRES_BLOCK8 : 1, 0};
  }
  py::tuple pair() const { return py::make_tuple(codes, scales); }
};

py::object quantize_8bit(const at::Tensor& X, bool tiles, bool rows, bool columns, uintptr_t stream) {
  const aires_dense x = dense(X, "X");
  New8 q, t;
  if (rows) q = New8(x.nrows, x.ncols, tiles, X.options());
  if (columns) t = New8(x.ncols, x.nrows, tiles, X.options());
  check(aires_quantize8(&x, rows ? &q.q : nullptr, columns ? &t.q : nullptr, (void*)stream), "aires_quantize8");
  if (!columns) return q.pair();
  if (!rows) return t.pair();
  return py::make_tuple(q.pair(), t.pair());
}

at::Tensor matmul_8bit(const py::tuple& A, const py::tuple& B, std::optional<at::ScalarType> out_dtype, const Maybe& out,
                       uintptr_t stream) {
  const at::Tensor &ac = part(A, 0, "A"), &as = part(A, 1, "A"), &bc = part(B, 0, "B"), &bs = part(B, 1, "B");
  const aires_dense8 a = held(ac, as, 1, "A"), b = held(bc, bs, 0, "B");
  if (a.ncols != b.ncols) bad_value("A and B differ in columns");
  same_device(ac, bc);
  if (out) same_device(ac, *out);
  if (out && out_dtype && out->scalar_type() != *out_dtype) throw py::type_error("out has another type than out_dtype");
  const at::Tensor Y = out ? *out : at::empty({a.nrows, b.nrows}, ac.options().dtype(out_dtype.value_or(at::kBFloat16)));
  const aires_dense y = dense(Y, "out");
  if (y.nrows != a.nrows || y.ncols != b.nrows) bad_value("out must have A's rows and a column for each of B's");
  int64_t need = 0;
  check(aires_matmul8_workspace(&a, &b, y.dtype, &need), "aires_matmul8_workspace");
  at::Tensor work;
  if (need > 0) work = at::empty({need}, ac.options().dtype(at::kByte));
  check(aires_matmul8(&a, &b, &y, need > 0 ? work.data_ptr() : nullptr, need, (void*)stream), "aires_matmul8");
  if (out) written(*out);
  return Y;
}

py::tuple rms_norm(const at::Tensor& X, const Maybe& gamma, const Maybe& residual, double eps,
                   std::optional<at::ScalarType> out_dtype, bool stats, const Maybe& out, const Maybe& sum_out,
                   uintptr_t stream) {
  const aires_dense x = dense(X, "X");
  const int64_t m = x.nrows, n = x.ncols;
  const void* g = gamma ? vector(*gamma, n, "gamma") : nullptr;
  const int32_t wt = gamma ? dtype_of(gamma->scalar_type()) : (int32_t)AIRES_F32;
  if (gamma) same_device(X, *gamma);
  if (out && out_dtype && out->scalar_type() != *out_dtype) throw py::type_error("out has another type than out_dtype");
  if (sum_out && !residual) bad_value("sum_out without residual");
  at::Tensor S, Y, rstd;
  aires_dense r{}, s{}, y{};
  if (residual) {
    same_device(X, *residual);
    r = dense(*residual, "residual");
    if (r.nrows != m || r.ncols != n) bad_value("X and residual differ in size");
    if (sum_out) same_device(X, *sum_out);
    S = sum_out ? *sum_out : at::empty({m, n}, residual->options());
    s = dense(S, "sum_out");
    if (s.nrows != m || s.ncols != n) bad_value("X and sum_out differ in size");
  }
  if (stats) rstd = at::empty({m}, X.options().dtype(at::kFloat));
  const bool eight = !out && out_dtype && *out_dtype == kCodes;
  New8 q;
  if (eight) {
    q = New8(m, n, false, X.options());
  } else {
    if (out) same_device(X, *out);
    Y = out ? *out : at::empty({m, n}, X.options().dtype(out_dtype.value_or(X.scalar_type())));
    y = dense(Y, "out");
    if (y.nrows != m || y.ncols != n) bad_value("X and out differ in size");
  }
  // (an empty vector has no address: nothing is written then)
  check(aires_rms_norm(&x, residual ? &r : nullptr, g, wt, eps, residual ? &s : nullptr, eight ? nullptr : &y,
                       eight ? &q.q : nullptr, stats && m > 0 ? rstd.data_ptr<float>() : nullptr, (void*)stream),
        "aires_rms_norm");
  if (out) written(*out);
  if (sum_out) written(*sum_out);
  return py::make_tuple(eight ? py::object(q.pair()) : py::cast(Y), or_none(S), or_none(rstd));
}

py::tuple rms_norm_backward(const at::Tensor& dY, const at::Tensor& S, const at::Tensor& rstd, const Maybe& gamma,
                            const Maybe& dS, bool need_dx, bool need_weights, std::optional<at::ScalarType> dx_dtype,
                            uintptr_t stream) {
  const aires_dense dy = dense(dY, "dY"), x = dense(S, "S");
  const int64_t m = x.nrows, n = x.ncols;
  if (dy.nrows != m || dy.ncols != n) bad_value("dY and S differ in size");
  const void* g = gamma ? vector(*gamma, n, "gamma") : nullptr;
  const void* q = vector(rstd, m, "rstd");
  if (rstd.scalar_type() != at::kFloat) throw py::type_error("rstd must be float32");
  same_device(S, dY);
  same_device(S, rstd);
  if (gamma) same_device(S, *gamma);
  aires_dense ds{}, dx{};
  if (dS) {
    same_device(S, *dS);
    ds = dense(*dS, "dS");
    if (ds.nrows != m || ds.ncols != n) bad_value("dS and S differ in size");
  }
  const at::ScalarType w = gamma ? gamma->scalar_type() : at::kFloat;
  const int32_t wt = dtype_of(w);
  at::Tensor dX, dg, work;
  if (need_dx) {
    dX = at::empty({m, n}, S.options().dtype(dx_dtype.value_or(S.scalar_type())));
    dx = dense(dX, "dX");
  }
  int64_t need = 0;
  if (need_weights) {
    check(aires_rms_norm_workspace(m, n, &need), "aires_rms_norm_workspace");
    dg = at::empty({n}, S.options().dtype(w));
    work = at::empty({need}, S.options().dtype(at::kByte));
  }
  check(aires_rms_norm_backward(&dy, &x, (const float*)q, g, wt, dS ? &ds : nullptr, need_dx ? &dx : nullptr,
                                need_weights ? dg.data_ptr() : nullptr, need_weights ? work.data_ptr() : nullptr, need,
                                (void*)stream),
        "aires_rms_norm_backward");
  return py::make_tuple(or_none(dX), or_none(dg));
}

const void* labels_of(const at::Tensor& labels, int64_t t) {
  if (labels.scalar_type() != at::kInt && labels.scalar_type() != at::kLong)
    throw py::type_error("labels must be int32 or int64");
  return vector(labels, t, "labels");
}

py::tuple log_probs(const at::Tensor& Z, const Maybe& labels, int64_t top, bool with_rest, uintptr_t stream) {
  const aires_dense z = dense(Z, "Z");
  const int64_t t = z.nrows;
  if (top < 0 || top > AIRES_MAX_TOP) bad_value("top must be between 0 and " + std::to_string(AIRES_MAX_TOP));
  const void* y = labels ? labels_of(*labels, t) : nullptr;
  if (labels) same_device(Z, *labels);
  int64_t need = 0;
  check(aires_log_probs_workspace(t, z.ncols, (int32_t)top, &need), "aires_log_probs_workspace");
  const at::TensorOptions f = Z.options().dtype(at::kFloat);
  at::Tensor work, logp, entropy = at::empty({t}, f), lse = at::empty({t}, f), rest, top_logp, top_index;
  if (need > 0) work = at::empty({need}, Z.options().dtype(at::kByte));
  if (labels) logp = at::empty({t}, f);
  if (with_rest) rest = at::empty({t}, f);
  if (top > 0) {
    top_logp = at::empty({t, top}, f);
    top_index = at::empty({t, top}, Z.options().dtype(at::kLong));
  }
  check(aires_log_probs_rest(&z, y, labels && labels->scalar_type() == at::kLong, (int32_t)top,
                             labels ? (float*)logp.data_ptr() : nullptr, (float*)entropy.data_ptr(),
                             (float*)lse.data_ptr(), with_rest ? (float*)rest.data_ptr() : nullptr,
                             top > 0 ? (float*)top_logp.data_ptr() : nullptr,
                             top > 0 ? (int64_t*)top_index.data_ptr() : nullptr,
                             need > 0 ? work.data_ptr() : nullptr, need, (void*)stream),
        "aires_log_probs");
  return py::make_tuple(or_none(logp), entropy, lse, or_none(top_logp), or_none(top_index), or_none(rest));
}

at::Tensor log_probs_backward(const at::Tensor& Z, const Maybe& labels, const at::Tensor& lse, const Maybe& lse_rest,
                              const Maybe& entropy, const Maybe& dlogp, const Maybe& dentropy,
                              std::optional<at::ScalarType> dz_dtype, const Maybe& out, uintptr_t stream) {
  const aires_dense z = dense(Z, "Z");
  const int64_t t = z.nrows;
  if (dlogp && !labels) bad_value("dlogp without labels");
  if (dentropy && !entropy) bad_value("dentropy without entropy");
  const auto numbers = [&](const at::Tensor& x, const char* name) {
    const void* p = vector(x, t, name);
    if (x.scalar_type() != at::kFloat) throw py::type_error(std::string(name) + " must be float32");
    same_device(Z, x);
    return (const float*)p;
  };
  const void* y = labels ? labels_of(*labels, t) : nullptr;
  if (labels) same_device(Z, *labels);
  const float *l = numbers(lse, "lse"), *lr = lse_rest ? numbers(*lse_rest, "lse_rest") : nullptr;
  const float *h = entropy ? numbers(*entropy, "entropy") : nullptr;
  const float *da = dlogp ? numbers(*dlogp, "dlogp") : nullptr, *db = dentropy ? numbers(*dentropy, "dentropy") : nullptr;
  if (out) same_device(Z, *out);
  if (out && dz_dtype && out->scalar_type() != *dz_dtype) throw py::type_error("out has another type than dz_dtype");
  const at::Tensor dZ = out ? *out : at::empty({t, z.ncols}, Z.options().dtype(dz_dtype.value_or(Z.scalar_type())));
  const aires_dense dz = dense(dZ, "out");
  if (dz.nrows != t || dz.ncols != z.ncols) bad_value("Z and out differ in size");
  check(aires_log_probs_backward_rest(&z, y, labels && labels->scalar_type() == at::kLong, l, lr, h, da, db, &dz,
                                      (void*)stream),
        "aires_log_probs_backward");
  if (out) written(*out);
  return dZ;
}

const at::Tensor& tensor(py::handle x) {
  if (!THPVariable_Check(x.ptr())) throw py::type_error("expected tensors");
  return THPVariable_Unpack(x.ptr());
}

// Gradients and where they go (outs: None for a norm alone).
std::vector<aires_grad_tensor> grad_table(const py::sequence& grads, const py::object& outs, at::Tensor& first) {
  const size_t n = grads.size();
  if (n == 0) bad_value("no gradients");
  const bool with = !outs.is_none();
  const py::sequence o = with ? py::reinterpret_borrow<py::sequence>(outs) : py::sequence();
  if (with && o.size() != n) bad_value("grads and out differ in number");
  std::vector<aires_grad_tensor> table(n);
  for (size_t k = 0; k < n; ++k) {
    const py::object go = grads[k];
    const at::Tensor& g = tensor(go);
    if (k == 0) {
      first = g;
      if (!g.is_cuda()) bad_value("gradients must be on a device");
    }
    if (!g.is_contiguous()) bad_value("gradient " + std::to_string(k) + " must be contiguous");
    same_device(first, g);
    aires_grad_tensor& t = table[k];
    t = aires_grad_tensor{g.numel(), g.data_ptr(), nullptr, dtype_of(g.scalar_type()), 0};
    if (with) {
      const py::object x = o[k];
      const at::Tensor& out = tensor(x);
      if (out.sizes() != g.sizes() || !out.is_contiguous())
        bad_value("out " + std::to_string(k) + " must be contiguous and of its gradient's shape");
      same_device(first, out);
      t.out = out.data_ptr();
      t.out_dtype = dtype_of(out.scalar_type());
    }
  }
  return table;
}

at::Tensor norm_workspace(int64_t count, const at::Tensor& first) {
  int64_t need = 0;
  check(aires_grad_norm_workspace(count, &need), "aires_grad_norm_workspace");
  return at::empty({need}, first.options().dtype(at::kByte));
}

py::tuple grad_norm(const py::sequence& grads, double max_norm, uintptr_t stream) {
  at::Tensor first;
  const auto table = grad_table(grads, py::none(), first);
  const at::Tensor work = norm_workspace((int64_t)table.size(), first);
  const at::Tensor norm = at::empty({}, first.options().dtype(at::kFloat)), scale = at::empty_like(norm);
  check(aires_grad_norm(table.data(), (int64_t)table.size(), max_norm, norm.data_ptr<float>(), scale.data_ptr<float>(),
                        work.data_ptr(), work.numel(), (void*)stream),
        "aires_grad_norm");
  return py::make_tuple(norm, scale);
}

at::Tensor clip_grads(const py::sequence& grads, const py::sequence& outs, double max_norm, uintptr_t stream) {
  at::Tensor first;
  const auto table = grad_table(grads, outs, first);
  const at::Tensor work = norm_workspace((int64_t)table.size(), first);
  const at::Tensor norm = at::empty({}, first.options().dtype(at::kFloat));
  check(aires_clip_grads(table.data(), (int64_t)table.size(), max_norm, norm.data_ptr<float>(), work.data_ptr(),
                         work.numel(), (void*)stream),
        "aires_clip_grads");
  for (size_t k = 0; k < table.size(); ++k) {
    const py::object x = outs[k];
    written(tensor(x));
  }
  return norm;
}

// One moment of parameter p: its address and that of its scales.
void moment(py::handle x, const at::Tensor& p, at::ScalarType codes_type, void*& at_, float*& scales_) {
  if (!PyTuple_Check(x.ptr())) {
    const at::Tensor& t = tensor(x);
    if (t.scalar_type() != at::kFloat || t.sizes() != p.sizes() || !t.is_contiguous() || t.device() != p.device())
      bad_value("expected contiguous float32 moments of the parameter's shape, on its device");
    at_ = t.data_ptr();
    scales_ = nullptr;
    return;
  }
  if (PyTuple_GET_SIZE(x.ptr()) != 2) bad_value("an 8-bit moment is a pair of codes and scales");
  const at::Tensor& codes = tensor(PyTuple_GET_ITEM(x.ptr(), 0));
  const at::Tensor& scales = tensor(PyTuple_GET_ITEM(x.ptr(), 1));
  if (codes.scalar_type() != codes_type || codes.sizes() != p.sizes() || !codes.is_contiguous() ||
      codes.device() != p.device())
    bad_value(std::string("expected contiguous ") + c10::toString(codes_type) + " codes of the parameter's shape, on its device");
  if (scales.scalar_type() != at::kFloat || !scales.is_contiguous() || scales.device() != p.device() ||
      scales.numel() != (p.numel() + AIRES_ADAMW_BLOCK - 1) / AIRES_ADAMW_BLOCK)
    bad_value("expected one float32 scale for each " + std::to_string(AIRES_ADAMW_BLOCK) + " values");
  at_ = codes.data_ptr();
  scales_ = (float*)scales.data_ptr();
}

void adamw(const py::sequence& params, const py::sequence& grads, const py::sequence& m, const py::sequence& v,
           const py::object& copies, int64_t step, double lr, double beta1, double beta2, double eps,
           double weight_decay, const py::object& grad_scale, uint32_t seed, uintptr_t stream) {
  const size_t n = params.size();
  const bool with = !copies.is_none();
  const py::sequence c = with ? py::reinterpret_borrow<py::sequence>(copies) : py::sequence();
  if (grads.size() != n || m.size() != n || v.size() != n || (with && c.size() != n))
    bad_value("params, grads, moments and copies differ in number");
  if (n == 0) return;
  std::vector<aires_adamw_tensor> table(n);
  const py::object first = params[0];
  const at::Device device = tensor(first).device();
  if (!device.is_cuda()) bad_value("parameters must be on a device");
  for (size_t k = 0; k < n; ++k) {
    const py::object po = params[k], go = grads[k], mo = m[k], vo = v[k];
    const at::Tensor &p = tensor(po), &g = tensor(go);
    if (g.sizes() != p.sizes() || !p.is_contiguous() || !g.is_contiguous())
      bad_value("parameter " + std::to_string(k) + " and its gradient must be contiguous and of one shape");
    if (p.device() != device || g.device() != device) bad_value("all tensors must be on one device");
    aires_adamw_tensor& t = table[k];
    t = aires_adamw_tensor{};
    t.n = p.numel();
    t.param = p.data_ptr();
    t.grad = g.data_ptr();
    t.param_dtype = dtype_of(p.scalar_type());
    t.grad_dtype = dtype_of(g.scalar_type());
    moment(mo, p, at::kFloat8_e4m3fn, t.exp_avg, t.exp_avg_scale);
    moment(vo, p, at::kFloat8_e5m2, t.exp_avg_sq, t.exp_avg_sq_scale);
    if (with) {
      const py::object co = c[k];
      if (!co.is_none()) {
        const at::Tensor& x = tensor(co);
        if (x.sizes() != p.sizes() || !x.is_contiguous() || x.device() != device)
          bad_value("copy " + std::to_string(k) + " must be contiguous and of its parameter's shape");
        t.copy = x.data_ptr();
        t.copy_dtype = dtype_of(x.scalar_type());
      }
    }
  }
  // One fp32 value on the parameters' device is read when the kernels run; all else that
  // has a float value, tensors too, now.
  const float* factor = nullptr;
  double number = 1.0;
  if (THPVariable_Check(grad_scale.ptr())) {
    const at::Tensor& x = THPVariable_Unpack(grad_scale.ptr());
    if (x.numel() != 1) throw py::type_error("grad_scale must be a number or a tensor of one value");
    if (x.scalar_type() == at::kFloat && x.device() == device) factor = (const float*)x.data_ptr();
  }
  if (!factor) {
    number = PyFloat_AsDouble(grad_scale.ptr());
    if (number == -1.0 && PyErr_Occurred()) throw py::error_already_set();
  }
  const aires_adamw_opts o{sizeof(aires_adamw_opts), seed, step, lr, beta1, beta2, eps, weight_decay, number};
  check(aires_adamw_scaled(table.data(), (int64_t)n, &o, factor, (void*)stream), "aires_adamw");
  for (size_t k = 0; k < n; ++k) {
    const py::object po = params[k], mo = m[k], vo = v[k];
    written(tensor(po));
    for (const py::handle x : {mo.ptr(), vo.ptr()})
      if (!PyTuple_Check(x.ptr())) written(tensor(x));
      else
        for (int i = 0; i < 2; ++i) written(tensor(PyTuple_GET_ITEM(x.ptr(), i)));
    if (table[k].copy) {
      const py::object co = c[k];
      written(tensor(co));
    }
  }
}

}  // namespace

PYBIND11_MODULE(TORCH_EXTENSION_NAME, m) {
  m.def("set_error", [](py::object e) { g_error = std::move(e); });
  m.def("abi_version", [] { return aires_abi_version(); });
  m.def("layer_norm", &layer_norm);
  m.def("layer_norm_backward", &layer_norm_backward);
  m.def("linear_xent", &linear_xent);
  m.def("adamw", &adamw);
  m.def("grad_norm", &grad_norm);
  m.def("clip_grads", &clip_grads);
  m.def("quantize_8bit", &quantize_8bit);
  m.def("matmul_8bit", &matmul_8bit);
  m.def("rms_norm", &rms_norm);
  m.def("rms_norm_backward", &rms_norm_backward);
  m.def("log_probs", &log_probs);
  m.def("log_probs_backward", &log_probs_backward);
  // the error class goes before the interpreter does
  m.add_object("_cleanup", py::capsule(+[] { g_error.release(); }));
}
