// binding_residual.cpp -- the calls on torch tensors of the operators between a block's
// products and of the product in 8-bit integers; as binding_block.cpp does it.
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>

#include "binding_args.h"
#include "fewbit_residual.h"

namespace {

using namespace binding;

// p, the seed (a number, or an int64 tensor of one element on ref's device) and the site.
struct Drop {
  fewbit_drop d{};
  at::Tensor seed;
  bool some = false;        // elements are dropped
};

// The place of a seed's ordinary device tensor.
const int64_t* seed_of(const at::Tensor& seed, const at::Tensor& ref) {
  TORCH_CHECK_TYPE(seed.scalar_type() == at::kLong, "seed must be a whole number or an int64 tensor");
  TORCH_CHECK_VALUE(seed.numel() == 1 && seed.device() == ref.device(), "a seed's tensor must have one element and be on the data's device");
  return seed.data_ptr<int64_t>();
}

Drop drop_of(PyObject* const* args, const at::Tensor& ref) {
  Drop r;
  r.d.p = number(args[0], "p");
  TORCH_CHECK_VALUE(r.d.p >= 0.0 && r.d.p <= 1.0, "p must be between 0 and 1");
  r.some = std::nearbyint(r.d.p * 65536.0) > 0.0;
  if (THPVariable_Check(args[1])) {
    r.seed = tensor(args[1], "seed");
    r.d.seed_at = seed_of(r.seed, ref);
  } else {
    // of either sign, or above 2^63
    const unsigned long long above = PyLong_Check(args[1]) ? PyLong_AsUnsignedLongLong(args[1]) : 0;
    const bool unsigned64 = PyLong_Check(args[1]) && !PyErr_Occurred();
    PyErr_Clear();
    r.d.seed = unsigned64 ? static_cast<int64_t>(above) : whole(args[1], "seed");
  }
  const int64_t site = whole(args[2], "site");
  TORCH_CHECK_VALUE(site >= 0 && site < int64_t{1} << 32, "site must be a whole number of 32 bits");
  r.d.site = static_cast<uint32_t>(site);
  return r;
}

// x with elements dropped; x as check_dense has it.
at::Tensor run_dropout(const at::Tensor& x, const fewbit_drop& d, int& rc) {
  at::AutoDispatchBelowADInplaceOrView below;
  const c10::DeviceGuard guard(x.device());
  at::Tensor y = at::empty(x.sizes(), x.options());
  rc = fewbit_dropout(&d, storage_type(x), x.numel(), x.data_ptr(), y.data_ptr(), stream_of(x));
  return y;
}

// dropout(x, p, seed, site) -> y, or a status
PyObject* dropout(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 4, "dropout takes four arguments");
  check_mode();
  const at::Tensor& x = tensor(args[0], "x");
  TORCH_CHECK_TYPE(storage_type(x) >= 0, "x must be float32, float16 or bfloat16");
  check_dense(x, "x");
  const Drop p = drop_of(args + 1, x);
  at::Tensor y;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    y = run_dropout(x, p.d, rc);
  }
  return rc == FEWBIT_OK ? THPVariable_Wrap(y) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// Sizes of rows [..., width]: rows of the last axis but one, `outer` of the axes before.
void rows_of(const at::Tensor& t, fewbit_rnorm& a) {
  const int64_t n = t.dim(), per = n > 0 ? t.size(n - 1) : 0;
  TORCH_CHECK_VALUE(n >= 1 && per >= 8 && per % 8 == 0 && per <= FEWBIT_RNORM_MOST, "rows must have a multiple of 8 elements up to ",
                    FEWBIT_RNORM_MOST);
  a.width = static_cast<int32_t>(per);
  a.rows = n > 1 ? t.size(n - 2) : 1;
  a.outer = 1;
  for (int64_t i = 0; i + 2 < n; ++i) a.outer *= t.size(i);
  TORCH_CHECK_VALUE(a.rows < int64_t{1} << 31 && a.outer < int64_t{1} << 31 && (a.rows == 0 || a.outer < ((int64_t{1} << 31) / a.rows)),
                    "there must be fewer than 2^31 rows");
}

// Strides {outer, row}, or false; the axes before the last two have to be one.
bool strides_fit(const at::Tensor& t, int64_t (&s)[2]) {
  const int64_t per = 16 / t.element_size(), n = t.dim();
  bool fits = reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0 && (t.size(n - 1) <= 1 || t.stride(n - 1) == 1);
  s[1] = n > 1 && t.size(n - 2) > 1 ? t.stride(n - 2) : 0;
  s[0] = 0;
  int64_t next = -1;        // the stride that the axis before would have
  for (int64_t i = n - 3; i >= 0; --i) {
    if (t.size(i) <= 1) continue;
    if (next < 0)
      s[0] = t.stride(i);
    else
      fits = fits && t.stride(i) == next;
    next = t.stride(i) * t.size(i);
  }
  for (const int64_t v : s) fits = fits && v % per == 0;
  return fits || t.numel() == 0;
}
void strides_of(const at::Tensor& t, const char* name, int64_t (&s)[2]) {
  TORCH_CHECK_VALUE(strides_fit(t, s), name, " must have contiguous rows that start at multiples of 16 bytes, in at most two even steps");
}

float eps_of(PyObject* o) {
  const double eps = number(o, "eps");
  TORCH_CHECK_VALUE(eps >= 0.0 && std::isfinite(static_cast<float>(eps)), "eps must be finite and not negative");
  return static_cast<float>(eps);
}

void check_weight(const at::Tensor& w, const at::Tensor& ref, const char* ref_name) {
  check_same(w, "weight", ref, ref_name);
  check_shape(w, "weight", {ref.size(-1)});
  check_dense(w, "weight");
}

fewbit_rnorm forward_of(const at::Tensor& x, const at::Tensor& residual, const at::Tensor& w, PyObject* eps) {
  fewbit_rnorm a{};
  TORCH_CHECK_TYPE(storage_type(x) >= 0, "x must be float32, float16 or bfloat16");
  rows_of(x, a);
  check_weight(w, x, "x");
  a.dtype = storage_type(x);
  a.eps = eps_of(eps);
  strides_of(x, "x", a.x_stride);
  if (residual.defined()) {
    check_same(residual, "residual", x, "x");
    check_shape(residual, "residual", x.sizes());
    strides_of(residual, "residual", a.residual_stride);
  }
  return a;
}

struct Sum {
  at::Tensor h, y;
};
Sum run_rnorm(const fewbit_rnorm& a, const at::Tensor& x, const at::Tensor& residual, const at::Tensor& w, bool sums, int& rc) {
  at::AutoDispatchBelowADInplaceOrView below;
  const c10::DeviceGuard guard(x.device());
  Sum r{sums ? at::empty(x.sizes(), x.options()) : x, at::empty(x.sizes(), x.options())};
  rc = fewbit_rnorm_fwd(&a, x.data_ptr(), pointer(residual), w.data_ptr(), sums ? r.h.data_ptr() : nullptr, r.y.data_ptr(), stream_of(x));
  return r;
}

// rnorm_fwd(x, residual, weight, eps, p, seed, site) -> (h, y), or a status; h is x where nothing is added or dropped
PyObject* rnorm_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 7, "rnorm_fwd takes seven arguments");
  check_mode();
  const at::Tensor &x = tensor(args[0], "x"), &w = tensor(args[2], "weight");
  const at::Tensor residual = optional(args[1], "residual");
  fewbit_rnorm a = forward_of(x, residual, w, args[3]);
  const Drop p = drop_of(args + 4, x);
  a.drop = p.d;
  Sum r;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    r = run_rnorm(a, x, residual, w, residual.defined() || p.some, rc);
  }
  return rc == FEWBIT_OK ? tuple_of(r.h, r.y) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// Scales of rows: x's shape without the last axis.
at::IntArrayRef lead_of(const at::Tensor& x) { return x.sizes().slice(0, x.dim() - 1); }

// rnorm_int8(x, residual, weight, eps) -> (h, codes, scale), or a status
PyObject* rnorm_int8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 4, "rnorm_int8 takes four arguments");
  check_mode();
  const at::Tensor &x = tensor(args[0], "x"), &w = tensor(args[2], "weight");
  const at::Tensor residual = optional(args[1], "residual");
  const fewbit_rnorm a = forward_of(x, residual, w, args[3]);
  at::Tensor h = x, codes, scale;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(x.device());
    if (residual.defined()) h = at::empty(x.sizes(), x.options());
    codes = at::empty(x.sizes(), x.options().dtype(at::kChar));
    scale = at::empty(lead_of(x), x.options().dtype(at::kFloat));
    rc = fewbit_rnorm_int8(&a, x.data_ptr(), pointer(residual), w.data_ptr(), residual.defined() ? h.data_ptr() : nullptr,
                           codes.data_ptr<int8_t>(), scale.data_ptr<float>(), stream_of(x));
  }
  return rc == FEWBIT_OK ? tuple_of(h, codes, scale) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// rows8(x) -> (codes, scale), or a status
PyObject* rows8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 1, "rows8 takes one argument");
  check_mode();
  const at::Tensor& x = tensor(args[0], "x");
  fewbit_rnorm a{};
  TORCH_CHECK_TYPE(storage_type(x) >= 0, "x must be float32, float16 or bfloat16");
  rows_of(x, a);
  a.dtype = storage_type(x);
  strides_of(x, "x", a.x_stride);
  at::Tensor codes, scale;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(x.device());
    codes = at::empty(x.sizes(), x.options().dtype(at::kChar));
    scale = at::empty(lead_of(x), x.options().dtype(at::kFloat));
    rc = fewbit_rows8(&a, x.data_ptr(), codes.data_ptr<int8_t>(), scale.data_ptr<float>(), stream_of(x));
  }
  return rc == FEWBIT_OK ? tuple_of(codes, scale) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

struct Gradients {
  at::Tensor dx, dres, dw;
};
Gradients run_rnorm_bwd(const fewbit_rnorm& a, const at::Tensor& dh, const at::Tensor& dy, const at::Tensor& h, const at::Tensor& w, bool apart,
                        int& rc) {
  at::AutoDispatchBelowADInplaceOrView below;
  const c10::DeviceGuard guard(h.device());
  Gradients g{at::empty(h.sizes(), h.options()), apart ? at::empty(h.sizes(), h.options()) : at::Tensor(),
              at::empty(w.sizes(), a.dw_dtype == a.dtype ? w.options() : w.options().dtype(at::kFloat))};
  const int64_t need = fewbit_rnorm_workspace(&a);
  const at::Tensor work = bytes(need, h);
  rc = need < 0 ? static_cast<int>(need)
                : fewbit_rnorm_bwd(&a, pointer(dh), dy.data_ptr(), h.data_ptr(), w.data_ptr(), g.dx.data_ptr(), pointer(g.dres), g.dw.data_ptr(),
                                   pointer(work), need, stream_of(h));
  return g;
}

// rnorm_bwd(dh, dy, h, weight, eps, p, seed, site, residual, rounded) -> (dx, dresidual, dweight), or a status.
// dresidual is dx where nothing is dropped, None where it is not asked for; dweight is fp32, or, rounded, of
// weight's type.
PyObject* rnorm_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 10, "rnorm_bwd takes ten arguments");
  check_mode();
  const at::Tensor dh = optional(args[0], "dh");
  const at::Tensor &dy = tensor(args[1], "dy"), &h = tensor(args[2], "h"), &w = tensor(args[3], "weight");
  fewbit_rnorm a{};
  TORCH_CHECK_TYPE(storage_type(h) >= 0, "h must be float32, float16 or bfloat16");
  rows_of(h, a);
  check_dense(h, "h");
  check_weight(w, h, "h");
  a.dtype = storage_type(h);
  a.eps = eps_of(args[4]);
  const Drop p = drop_of(args + 5, h);
  a.drop = p.d;
  const bool apart = truth(args[8], "residual") && p.some;
  if (truth(args[9], "rounded")) a.dw_dtype = a.dtype;
  check_same(dy, "dy", h, "h");
  check_shape(dy, "dy", h.sizes());
  strides_of(dy, "dy", a.dy_stride);
  if (dh.defined()) {
    check_same(dh, "dh", h, "h");
    check_shape(dh, "dh", h.sizes());
    strides_of(dh, "dh", a.dh_stride);
  }
  Gradients g;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    g = run_rnorm_bwd(a, dh, dy, h, w, apart, rc);
  }
  if (rc != FEWBIT_OK) return PyLong_FromLong(rc);
  if (!p.some) g.dres = g.dx;
  THPObjectPtr r(PyTuple_New(3));
  if (!r) return nullptr;
  const at::Tensor* items[] = {&g.dx, &g.dres, &g.dw};
  for (int i = 0; i < 3; ++i) {
    PyObject* o = items[i]->defined() ? THPVariable_Wrap(*items[i]) : Py_NewRef(Py_None);
    if (!o) return nullptr;
    PyTuple_SET_ITEM(r.get(), i, o);
  }
  return r.release();
  END_HANDLE_TH_ERRORS
}

// mm8(x, x_scale, weight, weight_scale, bias, act, dtype) -> y, or a status; dtype is that of the C ABI
PyObject* mm8(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 7, "mm8 takes seven arguments");
  check_mode();
  const at::Tensor &x = tensor(args[0], "x"), &xs = tensor(args[1], "x_scale"), &w = tensor(args[2], "weight"), &ws = tensor(args[3], "weight_scale");
  const at::Tensor bias = optional(args[4], "bias");
  fewbit_mm8 a{};
  a.act = static_cast<int32_t>(whole(args[5], "act"));
  a.dtype = static_cast<int32_t>(whole(args[6], "dtype"));
  constexpr at::ScalarType kTypes[] = {at::kFloat, at::kHalf, at::kBFloat16};
  TORCH_CHECK_TYPE(a.dtype >= 0 && a.dtype < 3, "y must be float32, float16 or bfloat16");
  TORCH_CHECK_TYPE(x.scalar_type() == at::kChar && w.scalar_type() == at::kChar, "x and weight must be int8");
  TORCH_CHECK_TYPE(xs.scalar_type() == at::kFloat && ws.scalar_type() == at::kFloat, "scales must be float32");
  TORCH_CHECK_VALUE(x.dim() >= 1 && w.dim() == 2 && x.size(-1) == w.size(1), "x is [..., width] and weight [out, width]");
  const int64_t width = w.size(1);
  TORCH_CHECK_VALUE(width >= 16 && width <= 131056 && width % 16 == 0, "width must be a multiple of 16 up to 131056");
  check_shape(xs, "x_scale", lead_of(x));
  check_shape(ws, "weight_scale", {w.size(0)});
  for (const auto& t : {w, xs, ws}) TORCH_CHECK_VALUE(t.device() == x.device(), "all tensors must be on x's device");
  check_dense(xs, "x_scale");
  check_dense(ws, "weight_scale");
  if (bias.defined()) {
    TORCH_CHECK_VALUE(bias.device() == x.device(), "bias must be on x's device");
    TORCH_CHECK_TYPE(bias.scalar_type() == kTypes[a.dtype], "bias must have y's dtype");
    check_shape(bias, "bias", {w.size(0)});
    check_dense(bias, "bias");
  }
  a.width = static_cast<int32_t>(width);
  a.out = w.size(0);
  a.rows = x.numel() / width;
  TORCH_CHECK_VALUE(a.rows < int64_t{1} << 31 && a.out < int64_t{1} << 31, "there must be fewer than 2^31 rows and channels");
  // one step from row to row
  int64_t next = -1;
  bool fits = x.stride(-1) == 1 && w.stride(1) == 1 && reinterpret_cast<uintptr_t>(x.data_ptr()) % 16 == 0 &&
              reinterpret_cast<uintptr_t>(w.data_ptr()) % 16 == 0;
  for (int64_t i = x.dim() - 2; i >= 0; --i) {
    if (x.size(i) <= 1) continue;
    if (next < 0)
      a.x_stride = x.stride(i);
    else
      fits = fits && x.stride(i) == next;
    next = x.stride(i) * x.size(i);
  }
  a.w_stride = a.out > 1 ? w.stride(0) : 0;
  fits = fits && a.x_stride % 16 == 0 && a.w_stride % 16 == 0;
  TORCH_CHECK_VALUE(fits || a.rows == 0 || a.out == 0, "x and weight must have contiguous rows at even steps of a multiple of 16 bytes");
  TORCH_CHECK_VALUE(a.x_stride <= FEWBIT_MM8_STRIDE && a.w_stride <= FEWBIT_MM8_STRIDE, "rows of x and weight must be at most ", FEWBIT_MM8_STRIDE,
                    " bytes apart");
  at::Tensor y;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(x.device());
    std::vector<int64_t> shape(lead_of(x).vec());
    shape.push_back(a.out);
    y = at::empty(shape, x.options().dtype(kTypes[a.dtype]));
    const int64_t need = fewbit_mm8_workspace(&a);
    const at::Tensor work = bytes(need, x);
    rc = need < 0 ? static_cast<int>(need)
                  : fewbit_mm8_fwd(&a, x.data_ptr<int8_t>(), xs.data_ptr<float>(), w.data_ptr<int8_t>(), ws.data_ptr<float>(), pointer(bias),
                                   y.data_ptr(), pointer(work), need, stream_of(x));
  }
  return rc == FEWBIT_OK ? THPVariable_Wrap(y) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- layers
// The differentiable calls without Python between them, for ordinary tensors whose layout the
// kernels take; for everything else they return None before they have done anything, and the
// package's own functions take over (they also raise what a wrong argument raises).
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

bool ordinary(PyObject* o) {
  if (!THPVariable_CheckExact(o)) return false;
  const at::Tensor& t = THPVariable_Unpack(o);
  return plain(t) && storage_type(t) >= 0 && !t.is_inference() && !t._fw_grad(0).defined();
}
bool dense(const at::Tensor& t) { return t.is_contiguous() && reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0; }
at::Tensor made_dense(const at::Tensor& t) { return dense(t) ? t : t.clone(at::MemoryFormat::Contiguous); }

// A hook may have put anything in the place of a saved tensor, so what a backward takes is checked
// as the arguments of a call are.
void check_ordinary(at::ArrayRef<at::Tensor> all) {
  for (const at::Tensor& t : all) TORCH_CHECK_VALUE(!t.defined() || plain(t), "saved tensors and gradients must be ordinary device tensors");
}

// What a backward needs of the dropout; the seed's tensor, if it is one, is saved last.
void keep(AutogradContext* ctx, const fewbit_drop& d) {
  ctx->saved_data["p"] = d.p;
  ctx->saved_data["seed"] = d.seed;
  ctx->saved_data["site"] = static_cast<int64_t>(d.site);
}
fewbit_drop kept(AutogradContext* ctx, const at::Tensor& seed_at, const at::Tensor& ref) {
  check_ordinary({seed_at});
  return {ctx->saved_data["p"].toDouble(), ctx->saved_data["seed"].toInt(), seed_at.defined() ? seed_of(seed_at, ref) : nullptr,
          static_cast<uint32_t>(ctx->saved_data["site"].toInt()), 0};
}

struct DropoutFn : torch::autograd::Function<DropoutFn> {
  static at::Tensor forward(AutogradContext* ctx, const at::Tensor& x, const fewbit_drop* d, const at::Tensor* seed_at) {
    keep(ctx, *d);
    if (seed_at->defined()) ctx->save_for_backward({*seed_at});
    int rc;
    at::Tensor y = run_dropout(x, *d, rc);
    if (rc != FEWBIT_OK) throw_status(rc, "fewbit_dropout");
    return y;
  }
  // The same function of the gradient, to any order.
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    const variable_list saved = ctx->get_saved_variables();
    check_ordinary({grads[0]});
    const at::Tensor seed_at = saved.empty() ? at::Tensor() : saved[0], dy = made_dense(grads[0]);
    const fewbit_drop d = kept(ctx, seed_at, dy);
    at::Tensor dx;
    if (at::GradMode::is_enabled()) {
      dx = apply(dy, &d, &seed_at);
    } else {
      int rc;
      dx = run_dropout(dy, d, rc);
      if (rc != FEWBIT_OK) throw_status(rc, "fewbit_dropout");
    }
    return {dx, at::Tensor(), at::Tensor()};
  }
};

// dropout_layer(x, p, seed, site) -> y with its history, or None
PyObject* dropout_layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 4 || !plain_mode() || !ordinary(args[0]) || !dense(THPVariable_Unpack(args[0]))) Py_RETURN_NONE;
  const at::Tensor& x = THPVariable_Unpack(args[0]);
  const Drop p = drop_of(args + 1, x);
  at::Tensor y;
  {
    pybind11::gil_scoped_release no_gil;
    y = DropoutFn::apply(x, &p.d, &p.seed);
  }
  return THPVariable_Wrap(y);
  END_HANDLE_TH_ERRORS
}

struct ResidualNormFn : torch::autograd::Function<ResidualNormFn> {
  static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const std::optional<at::Tensor>& residual, const at::Tensor& w,
                               const fewbit_rnorm* a, const at::Tensor* seed_at) {
    int rc;
    const Sum r = run_rnorm(*a, x, residual.value_or(at::Tensor()), w, true, rc);
    if (rc != FEWBIT_OK) throw_status(rc, "fewbit_rnorm_fwd");
    keep(ctx, a->drop);
    ctx->saved_data["eps"] = static_cast<double>(a->eps);
    ctx->saved_data["residual"] = residual.has_value();        // else the weight is the second input
    variable_list saved{r.h, w};
    if (seed_at->defined()) saved.push_back(*seed_at);
    ctx->save_for_backward(std::move(saved));
    ctx->set_materialize_grads(false);
    return {r.h, r.y};
  }
  static variable_list backward(AutogradContext* ctx, variable_list grads) {
    variable_list none(5);
    if (!grads[0].defined() && !grads[1].defined()) return none;
    const variable_list saved = ctx->get_saved_variables();
    const at::Tensor &h = saved[0], &w = saved[1];
    at::Tensor dh = grads[0], dy = grads[1];
    check_ordinary({h, w, dh, dy});
    fewbit_rnorm a{};
    TORCH_CHECK_TYPE(storage_type(h) >= 0, "h must be float32, float16 or bfloat16");
    rows_of(h, a);
    a.dtype = a.dw_dtype = storage_type(h);
    a.eps = static_cast<float>(ctx->saved_data["eps"].toDouble());
    a.drop = kept(ctx, saved.size() > 2 ? saved[2] : at::Tensor(), h);
    check_same(w, "weight", h, "h");
    check_shape(w, "weight", {h.size(-1)});
    for (const at::Tensor& t : {dh, dy}) {
      if (!t.defined()) continue;
      check_same(t, "the gradient", h, "h");
      check_shape(t, "the gradient", h.sizes());
    }
    if (!dy.defined()) dy = at::zeros_like(h);
    if (dh.defined() && !strides_fit(dh, a.dh_stride)) {
      dh = dh.clone(at::MemoryFormat::Contiguous);
      strides_of(dh, "dh", a.dh_stride);
    }
    if (!strides_fit(dy, a.dy_stride)) {
      dy = dy.clone(at::MemoryFormat::Contiguous);
      strides_of(dy, "dy", a.dy_stride);
    }
    const bool some = std::nearbyint(a.drop.p * 65536.0) > 0.0, residual = ctx->saved_data["residual"].toBool() && ctx->needs_input_grad(1);
    int rc;
    Gradients g = run_rnorm_bwd(a, dh, dy, made_dense(h), made_dense(w), some && residual, rc);
    if (rc != FEWBIT_OK) throw_status(rc, "fewbit_rnorm_bwd");
    if (!some) g.dres = g.dx;
    variable_list out{g.dx, residual ? g.dres : at::Tensor(), g.dw, at::Tensor(), at::Tensor()};
    if (!at::GradMode::is_enabled()) return out;
    // gradients of these gradients are not formed: asking for them raises
    for (at::Tensor& t : out)
      if (t.defined()) t = t.detach().set_requires_grad(true);
    return std::make_shared<torch::autograd::DelayedError>("the gradient of residual_norm cannot be differentiated", static_cast<int64_t>(out.size()))
        ->operator()(std::move(out));
  }
};

// residual_norm_layer(x, residual, weight, eps, p, seed, site) -> (h, y) with their history, or None
PyObject* residual_norm_layer(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  if (nargs != 7 || !plain_mode() || !ordinary(args[0]) || !ordinary(args[2]) || (args[1] != Py_None && !ordinary(args[1]))) Py_RETURN_NONE;
  const at::Tensor &x = THPVariable_Unpack(args[0]), &w = THPVariable_Unpack(args[2]);
  const at::Tensor residual = args[1] == Py_None ? at::Tensor() : THPVariable_Unpack(args[1]);
  int64_t s[2];
  if (x.dim() < 1 || !strides_fit(x, s) || !dense(w) || (residual.defined() && (residual.dim() < 1 || !strides_fit(residual, s)))) Py_RETURN_NONE;
  fewbit_rnorm a = forward_of(x, residual, w, args[3]);
  const Drop p = drop_of(args + 4, x);
  if (!residual.defined() && !p.some) Py_RETURN_NONE;       // h is x
  a.drop = p.d;
  variable_list r;
  {
    pybind11::gil_scoped_release no_gil;
    r = ResidualNormFn::apply(x, residual.defined() ? std::optional<at::Tensor>(residual) : std::nullopt, w, &a, &p.seed);
  }
  return tuple_of(r[0], r[1]);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {method<dropout_layer>("dropout_layer"), method<residual_norm_layer>("residual_norm_layer"),
                         method<dropout>("dropout"), method<rnorm_fwd>("rnorm_fwd"), method<rnorm_bwd>("rnorm_bwd"),
                         method<rnorm_int8>("rnorm_int8"), method<rows8>("rows8"), method<mm8>("mm8"), {nullptr, nullptr, 0, nullptr}};

}  // namespace

PyMethodDef* binding::residual_methods() { return methods; }
