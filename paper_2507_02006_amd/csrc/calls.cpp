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
  const auto or_none = [](const at::Tensor& t) -> py::object { return t.defined() ? py::cast(t) : py::none(); };
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
  const auto or_none = [](const at::Tensor& t) -> py::object { return t.defined() ? py::cast(t) : py::none(); };
  return py::make_tuple(loss, rows, or_none(dH), or_none(dW));
}

const at::Tensor& tensor(py::handle x) {
  if (!THPVariable_Check(x.ptr())) throw py::type_error("expected tensors");
  return THPVariable_Unpack(x.ptr());
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
           double weight_decay, double grad_scale, uint32_t seed, uintptr_t stream) {
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
  const aires_adamw_opts o{sizeof(aires_adamw_opts), seed, step, lr, beta1, beta2, eps, weight_decay, grad_scale};
  check(aires_adamw(table.data(), (int64_t)n, &o, (void*)stream), "aires_adamw");
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
  // the error class goes before the interpreter does
  m.add_object("_cleanup", py::capsule(+[] { g_error.release(); }));
}
