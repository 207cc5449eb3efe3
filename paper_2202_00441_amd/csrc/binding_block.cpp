// binding_block.cpp -- the block operators' calls on torch tensors: checks of
// every tensor (device, type, shape, layout), allocation of the results and of
// the workspace, the current stream, and the call of the C ABI.
//
// A wrong argument raises TypeError or ValueError before anything is launched;
// a status of the library comes back as a number, which the package turns into
// its exception.
#include "binding_args.h"
#include "fewbit_block.h"

namespace {

using namespace binding;

// ---------------------------------------------------------------- attention
struct Attention {
  fewbit_attn a{};
  at::Tensor cu_q, cu_k, k_len;
};

// args: causal, window, scale or None, k_len, cu_q, cu_k
Attention attention_of(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, PyObject* const* args) {
  check_mode();
  Attention r;
  fewbit_attn& a = r.a;
  r.k_len = optional(args[3], "k_len");
  r.cu_q = optional(args[4], "cu_q");
  r.cu_k = optional(args[5], "cu_k");
  const bool packed = r.cu_q.defined();
  TORCH_CHECK_VALUE(packed == r.cu_k.defined(), "cu_q and cu_k go together");
  TORCH_CHECK_VALUE(!packed || !r.k_len.defined(), "k_len is for sequences that are not packed");
  TORCH_CHECK_TYPE(q.scalar_type() == at::kHalf || q.scalar_type() == at::kBFloat16, "q must be float16 or bfloat16");
  check_same(k, "k", q, "q");
  check_same(v, "v", q, "q");
  const int64_t n = packed ? 3 : 4;
  TORCH_CHECK_VALUE(q.dim() == n && k.dim() == n, packed ? "packed q, k and v are [rows, heads, head_dim]"
                                                         : "q, k and v are [batch, rows, heads, head_dim]");
  check_shape(v, "v", k.sizes());
  TORCH_CHECK_VALUE(k.size(n - 1) == q.size(n - 1) && (packed || k.size(0) == q.size(0)),
                    "k and v must have q's batch and head_dim");
  a.dtype = storage_type(q);
  a.heads_q = static_cast<int32_t>(q.size(n - 2));
  a.heads_kv = static_cast<int32_t>(k.size(n - 2));
  a.head_dim = static_cast<int32_t>(q.size(n - 1));
  TORCH_CHECK_VALUE(a.heads_kv > 0 && a.heads_q > 0 && a.heads_q % a.heads_kv == 0,
                    "q's heads must be a multiple of k's");
  TORCH_CHECK_VALUE(a.head_dim % 8 == 0 && a.head_dim >= 8 && a.head_dim <= 128, "head_dim must be a multiple of 8 up to 128");
  a.causal = truth(args[0], "causal");
  const int64_t window = whole(args[1], "window");
  TORCH_CHECK_VALUE(window >= 0 && window < int64_t{1} << 31, "window must not be negative");
  TORCH_CHECK_VALUE(window == 0 || a.causal, "window needs causal");
  a.window = static_cast<int32_t>(window);
  a.scale = static_cast<float>(args[2] == Py_None ? 1.0 / std::sqrt(static_cast<double>(a.head_dim)) : number(args[2], "scale"));
  TORCH_CHECK_VALUE(a.scale > 0.0f && std::isfinite(a.scale), "scale must be positive and finite");
  a.rows_q = q.size(n - 3);
  a.rows_k = k.size(n - 3);
  a.batch = packed ? r.cu_q.numel() - 1 : q.size(0);
  if (packed) {
    TORCH_CHECK_VALUE(a.batch >= 0, "cu_q and cu_k hold one more entry than there are sequences");
    for (const auto& t : {r.cu_q, r.cu_k}) {
      TORCH_CHECK_VALUE(t.scalar_type() == at::kInt && t.is_contiguous() && t.device() == q.device() && t.numel() == a.batch + 1,
                        "cu_q and cu_k must be contiguous int32 tensors of equal length on q's device");
    }
    a.cu_q = r.cu_q.data_ptr<int32_t>();
    a.cu_k = r.cu_k.data_ptr<int32_t>();
  }
  if (r.k_len.defined()) {
    TORCH_CHECK_VALUE(r.k_len.scalar_type() == at::kInt && r.k_len.is_contiguous() && r.k_len.device() == q.device() &&
                          r.k_len.numel() == a.batch,
                      "k_len must be a contiguous int32 tensor with an entry for each sequence on q's device");
    a.k_len = a.batch > 0 ? r.k_len.data_ptr<int32_t>() : nullptr;
  }
  strides_of(q, "q", a.q_stride);
  strides_of(k, "k", a.k_stride);
  strides_of(v, "v", a.v_stride);
  return r;
}

// Shape of lse: [batch, heads, rows] or, packed, [heads, rows].
std::vector<int64_t> lse_shape(const at::Tensor& q) {
  if (q.dim() == 3) return {q.size(1), q.size(0)};
  return {q.size(0), q.size(2), q.size(1)};
}

// attention_fwd(q, k, v, causal, window, scale, k_len, cu_q, cu_k) -> (out, lse), or a status
PyObject* attention_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 9, "attention_fwd takes nine arguments");
  const at::Tensor &q = tensor(args[0], "q"), &k = tensor(args[1], "k"), &v = tensor(args[2], "v");
  const Attention p = attention_of(q, k, v, args + 3);
  at::Tensor out, lse;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(q.device());
    out = at::empty(q.sizes(), q.options());
    lse = at::empty(lse_shape(q), q.options().dtype(at::kFloat));
    const int64_t need = fewbit_attn_workspace(&p.a, 0);
    const at::Tensor work = bytes(need, q);
    rc = need < 0 ? static_cast<int>(need)
                  : fewbit_attn_fwd(&p.a, q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr<float>(),
                                    pointer(work), need, stream_of(q));
  }
  return rc == FEWBIT_OK ? tuple_of(out, lse) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// attention_bwd(dout, q, k, v, out, lse, causal, window, scale, k_len, cu_q, cu_k) -> (dq, dk, dv), or a status
PyObject* attention_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 12, "attention_bwd takes twelve arguments");
  const at::Tensor &dout = tensor(args[0], "dout"), &q = tensor(args[1], "q"), &k = tensor(args[2], "k"),
                   &v = tensor(args[3], "v"), &out = tensor(args[4], "out"), &lse = tensor(args[5], "lse");
  Attention p = attention_of(q, k, v, args + 6);
  check_same(dout, "dout", q, "q");
  check_same(out, "out", q, "q");
  check_shape(dout, "dout", q.sizes());
  check_shape(out, "out", q.sizes());
  check_shape(lse, "lse", lse_shape(q));
  TORCH_CHECK_VALUE(lse.scalar_type() == at::kFloat && lse.device() == q.device(), "lse must be float32 on q's device");
  check_dense(out, "out");
  check_dense(lse, "lse");
  strides_of(dout, "dout", p.a.dout_stride);
  at::Tensor dq, dk, dv;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(q.device());
    dq = at::empty(q.sizes(), q.options());
    dk = at::empty(k.sizes(), k.options());
    dv = at::empty(v.sizes(), v.options());
    const int64_t need = fewbit_attn_workspace(&p.a, 1);
    const at::Tensor work = bytes(need, q);
    rc = need < 0 ? static_cast<int>(need)
                  : fewbit_attn_bwd(&p.a, dout.data_ptr(), q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(),
                                    lse.data_ptr<float>(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), pointer(work), need,
                                    stream_of(q));
  }
  return rc == FEWBIT_OK ? tuple_of(dq, dk, dv) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- norm and rotation
struct Qk {
  fewbit_qk a{};
  at::Tensor positions;
  const float *cos = nullptr, *sin = nullptr;
};

// args: q_weight, k_weight, cos, sin, positions, eps, interleaved
Qk qk_of(const at::Tensor& q, const at::Tensor& k, PyObject* const* args) {
  check_mode();
  Qk r;
  fewbit_qk& a = r.a;
  const int64_t n = q.dim();
  TORCH_CHECK_TYPE(storage_type(q) >= 0, "q must be float32, float16 or bfloat16");
  check_same(k, "k", q, "q");
  TORCH_CHECK_VALUE((n == 4 || n == 3) && k.dim() == n && q.size(n - 1) == k.size(n - 1) && q.size(n - 3) == k.size(n - 3) &&
                        (n == 3 || q.size(0) == k.size(0)),
                    "q and k are [batch, tokens, heads, head_dim] or [tokens, heads, head_dim], alike but for the heads");
  const int64_t d = q.size(n - 1);
  TORCH_CHECK_VALUE(d % 16 == 0 && d >= 16 && d <= 256, "head_dim must be a multiple of 16 up to 256");
  for (int i = 0; i < 2; ++i) {
    const char* name = i ? "k_weight" : "q_weight";
    const at::Tensor& w = tensor(args[i], name);
    check_same(w, name, q, "q");
    check_shape(w, name, {d});
    check_dense(w, name);
  }
  const at::Tensor &cos = tensor(args[2], "cos"), &sin = tensor(args[3], "sin");
  TORCH_CHECK_VALUE(cos.dim() == 2 && cos.sizes() == sin.sizes(), "cos and sin are [positions, rotated elements / 2]");
  for (const auto& t : {cos, sin}) {
    TORCH_CHECK_TYPE(t.scalar_type() == at::kFloat, "cos and sin must be float32");
    TORCH_CHECK_VALUE(t.device() == q.device(), "cos and sin must be on q's device");
    check_dense(t, "cos and sin");
  }
  const int64_t rot = 2 * cos.size(1);
  TORCH_CHECK_VALUE(rot % 16 == 0 && rot <= d, "the rotated part must be a multiple of 16 elements and no more than head_dim");
  r.cos = cos.data_ptr<float>();
  r.sin = sin.data_ptr<float>();
  a.dtype = storage_type(q);
  a.heads_q = static_cast<int32_t>(q.size(n - 2));
  a.heads_k = static_cast<int32_t>(k.size(n - 2));
  a.head_dim = static_cast<int32_t>(d);
  a.rot = static_cast<int32_t>(rot);
  a.batch = n == 4 ? q.size(0) : 1;
  a.tokens = q.size(n - 3);
  a.table_rows = cos.size(0);
  const at::Tensor positions = optional(args[4], "positions");
  if (positions.defined()) {
    TORCH_CHECK_TYPE(positions.scalar_type() == at::kLong, "positions must be int64");
    TORCH_CHECK_VALUE(positions.device() == q.device(), "positions must be on q's device");
    const bool one = positions.dim() == 1 && positions.size(0) == a.tokens;
    const bool two = n == 4 && positions.dim() == 2 && positions.size(1) == a.tokens &&
                     (positions.size(0) == a.batch || positions.size(0) == 1);
    TORCH_CHECK_VALUE(one || two, "positions must be [tokens] or [batch, tokens]");
    r.positions = positions;
    a.position_stride[0] = two && positions.size(0) > 1 ? positions.stride(0) : 0;
    a.position_stride[1] = positions.stride(-1);
  } else {
    TORCH_CHECK_VALUE(rot == 0 || a.tokens <= a.table_rows, "cos and sin must hold a row for every token");
  }
  const double eps = number(args[5], "eps");
  TORCH_CHECK_VALUE(eps >= 0.0 && std::isfinite(static_cast<float>(eps)), "eps must be finite and not negative");
  a.eps = static_cast<float>(eps);
  a.interleaved = truth(args[6], "interleaved");
  strides_of(q, "q", a.q_stride);
  strides_of(k, "k", a.k_stride);
  return r;
}

const int64_t* positions_of(const Qk& p) { return p.positions.defined() ? p.positions.data_ptr<int64_t>() : nullptr; }

// qk_fwd(q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved) -> (q, k), or a status
PyObject* qk_fwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 9, "qk_fwd takes nine arguments");
  const at::Tensor &q = tensor(args[0], "q"), &k = tensor(args[1], "k");
  const Qk p = qk_of(q, k, args + 2);
  const at::Tensor &qw = THPVariable_Unpack(args[2]), &kw = THPVariable_Unpack(args[3]);
  at::Tensor qo, ko;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(q.device());
    qo = at::empty(q.sizes(), q.options());
    ko = at::empty(k.sizes(), k.options());
    rc = fewbit_qk_fwd(&p.a, q.data_ptr(), k.data_ptr(), qw.data_ptr(), kw.data_ptr(), p.cos, p.sin, positions_of(p),
                       qo.data_ptr(), ko.data_ptr(), stream_of(q));
  }
  return rc == FEWBIT_OK ? tuple_of(qo, ko) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// qk_bwd(dq, dk, q, k, q_weight, k_weight, cos, sin, positions, eps, interleaved) -> (dq, dk, dq_weight, dk_weight), or a status
PyObject* qk_bwd(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 11, "qk_bwd takes eleven arguments");
  const at::Tensor &gq = tensor(args[0], "dq"), &gk = tensor(args[1], "dk"), &q = tensor(args[2], "q"), &k = tensor(args[3], "k");
  Qk p = qk_of(q, k, args + 4);
  const at::Tensor &qw = THPVariable_Unpack(args[4]), &kw = THPVariable_Unpack(args[5]);
  check_same(gq, "dq", q, "q");
  check_same(gk, "dk", q, "q");
  check_shape(gq, "dq", q.sizes());
  check_shape(gk, "dk", k.sizes());
  strides_of(gq, "dq", p.a.dq_stride);
  strides_of(gk, "dk", p.a.dk_stride);
  at::Tensor dq, dk, dqw, dkw;
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    at::AutoDispatchBelowADInplaceOrView below;
    const c10::DeviceGuard guard(q.device());
    dq = at::empty(q.sizes(), q.options());
    dk = at::empty(k.sizes(), k.options());
    dqw = at::empty(qw.sizes(), qw.options().dtype(at::kFloat));
    dkw = at::empty(kw.sizes(), kw.options().dtype(at::kFloat));
    const int64_t need = fewbit_qk_workspace(&p.a);
    const at::Tensor work = bytes(need, q);
    rc = need < 0 ? static_cast<int>(need)
                  : fewbit_qk_bwd(&p.a, gq.data_ptr(), gk.data_ptr(), q.data_ptr(), k.data_ptr(), qw.data_ptr(), kw.data_ptr(),
                                  p.cos, p.sin, positions_of(p), dq.data_ptr(), dk.data_ptr(), dqw.data_ptr<float>(),
                                  dkw.data_ptr<float>(), pointer(work), need, stream_of(q));
  }
  return rc == FEWBIT_OK ? tuple_of(dq, dk, dqw, dkw) : PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

// ---------------------------------------------------------------- AdamW
// A flat buffer of the optimizer: contiguous, aligned, long enough.
void check_flat(const at::Tensor& t, const char* name, const at::Tensor& ref, at::ScalarType type, int64_t n) {
  TORCH_CHECK_VALUE(t.device() == ref.device(), name, " must be on the parameters' device");
  TORCH_CHECK_TYPE(t.scalar_type() == type, name, " must have dtype ", type);
  TORCH_CHECK_VALUE(t.numel() >= n, name, " holds ", t.numel(), " elements, ", n, " are needed");
  check_dense(t, name);
}

// adamw_step(params, grads, m, v, m_scale, v_scale, master, lr, beta1, beta2, eps, weight_decay, step, seed) -> status
PyObject* adamw_step(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
  HANDLE_TH_ERRORS
  TORCH_CHECK_TYPE(nargs == 14, "adamw_step takes fourteen arguments");
  check_mode();
  THPObjectPtr params(PySequence_Fast(args[0], "params must be a sequence of tensors"));
  THPObjectPtr grads(PySequence_Fast(args[1], "grads must be a sequence of tensors"));
  if (!params || !grads) throw python_error();
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(params.get());
  TORCH_CHECK_VALUE(n == PySequence_Fast_GET_SIZE(grads.get()), "params and grads must have the same length");
  fewbit_adamw h{};
  h.lr = number(args[7], "lr");
  h.beta1 = number(args[8], "beta1");
  h.beta2 = number(args[9], "beta2");
  h.eps = number(args[10], "eps");
  h.weight_decay = number(args[11], "weight_decay");
  h.step = whole(args[12], "step");
  h.seed = whole(args[13], "seed");
  if (n == 0) return PyLong_FromLong(FEWBIT_OK);
  const at::Tensor& first = tensor(PySequence_Fast_GET_ITEM(params.get(), 0), "params");
  h.param_dtype = storage_type(first);
  TORCH_CHECK_TYPE(h.param_dtype >= 0, "params must be float32, float16 or bfloat16");
  h.grad_dtype = -1;
  std::vector<fewbit_adamw_tensor> list(n);
  int64_t blocks = 0;
  for (Py_ssize_t i = 0; i < n; ++i) {
    const at::Tensor& p = tensor(PySequence_Fast_GET_ITEM(params.get(), i), "params");
    check_same(p, "every parameter", first, "the first");
    TORCH_CHECK_VALUE(p.is_non_overlapping_and_dense(), "parameters must be dense");
    list[i] = {p.data_ptr(), nullptr, p.numel()};
    blocks += (p.numel() + FEWBIT_ADAMW_BLOCK - 1) / FEWBIT_ADAMW_BLOCK;
    PyObject* o = PySequence_Fast_GET_ITEM(grads.get(), i);
    if (o == Py_None) continue;
    const at::Tensor& g = tensor(o, "grads");
    TORCH_CHECK_VALUE(g.device() == p.device(), "every gradient must be on its parameter's device");
    const int gt = storage_type(g);
    TORCH_CHECK_TYPE(gt == h.param_dtype || gt == FEWBIT_F32, "gradients must have the parameters' dtype or float32");
    TORCH_CHECK_TYPE(h.grad_dtype < 0 || gt == h.grad_dtype, "gradients must all have the same dtype");
    h.grad_dtype = gt;
    TORCH_CHECK_VALUE(g.sizes() == p.sizes() && ((g.is_contiguous() && p.is_contiguous()) || g.strides() == p.strides()),
                      "every gradient must have its parameter's shape and layout");
    list[i].grad = g.data_ptr();
  }
  if (h.grad_dtype < 0) return PyLong_FromLong(FEWBIT_OK);         // no gradients
  const at::Tensor &m = tensor(args[2], "exp_avg"), &v = tensor(args[3], "exp_avg_sq");
  h.state_bits = m.scalar_type() == at::kFloat8_e4m3fn ? 8 : 32;
  const at::ScalarType state = h.state_bits == 8 ? at::kFloat8_e4m3fn : at::kFloat;
  check_flat(m, "exp_avg", first, state, blocks * FEWBIT_ADAMW_BLOCK);
  check_flat(v, "exp_avg_sq", first, state, blocks * FEWBIT_ADAMW_BLOCK);
  const at::Tensor ms = optional(args[4], "exp_avg_scale"), vs = optional(args[5], "exp_avg_sq_scale"), master = optional(args[6], "master");
  if (h.state_bits == 8) {
    TORCH_CHECK_VALUE(ms.defined() && vs.defined(), "moments in 8 bits need their scales");
    check_flat(ms, "exp_avg_scale", first, at::kFloat, blocks);
    check_flat(vs, "exp_avg_sq_scale", first, at::kFloat, blocks);
  }
  if (master.defined()) {
    TORCH_CHECK_VALUE(h.param_dtype != FEWBIT_F32, "float32 parameters have no master copy");
    check_flat(master, "master", first, at::kFloat, blocks * FEWBIT_ADAMW_BLOCK);
  }
  // autograd sees that they change
  for (Py_ssize_t i = 0; i < n; ++i)
    if (list[i].grad) changed(THPVariable_Unpack(PySequence_Fast_GET_ITEM(params.get(), i)));
  for (const auto& t : {m, v, ms, vs, master})
    if (t.defined()) changed(t);
  int rc;
  {
    pybind11::gil_scoped_release no_gil;
    const c10::DeviceGuard guard(first.device());
    rc = fewbit_adamw_step(&h, list.data(), static_cast<int32_t>(n), m.data_ptr(), v.data_ptr(),
                           static_cast<float*>(pointer(ms)), static_cast<float*>(pointer(vs)),
                           static_cast<float*>(pointer(master)), stream_of(first));
  }
  return PyLong_FromLong(rc);
  END_HANDLE_TH_ERRORS
}

PyMethodDef methods[] = {method<attention_fwd>("attention_fwd"), method<attention_bwd>("attention_bwd"),
                         method<qk_fwd>("qk_fwd"), method<qk_bwd>("qk_bwd"),
                         method<adamw_step>("adamw_step"), {nullptr, nullptr, 0, nullptr}};

}  // namespace

PyMethodDef* binding::block_methods() { return methods; }
