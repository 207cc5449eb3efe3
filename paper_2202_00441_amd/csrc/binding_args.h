// binding_args.h -- what the calls on torch tensors share beyond binding.h: their
// arguments and results.
#pragma once

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>
#include <torch/csrc/utils/pybind.h>

#include <c10/core/DeviceGuard.h>

#include <cmath>
#include <string>
#include <vector>

#include "binding.h"

namespace binding {

inline const at::Tensor& tensor(PyObject* o, const char* name) {
  TORCH_CHECK_TYPE(THPVariable_Check(o), name, " must be a tensor");
  const at::Tensor& t = THPVariable_Unpack(o);
  TORCH_CHECK_VALUE(plain(t), name, " must be an ordinary device tensor");
  return t;
}

// A tensor or None.
inline at::Tensor optional(PyObject* o, const char* name) { return o == Py_None ? at::Tensor() : tensor(o, name); }

inline void check_mode() {
  TORCH_CHECK_VALUE(plain_mode(), "not available while tensor operations are traced, transformed or dispatched elsewhere");
}

inline void check_same(const at::Tensor& t, const char* name, const at::Tensor& ref, const char* ref_name) {
  TORCH_CHECK_VALUE(t.device() == ref.device(), name, " must be on ", ref_name, "'s device");
  TORCH_CHECK_TYPE(t.scalar_type() == ref.scalar_type(), name, " must have ", ref_name, "'s dtype");
}

inline void check_shape(const at::Tensor& t, const char* name, at::IntArrayRef shape) {
  TORCH_CHECK_VALUE(t.sizes() == shape, name, " must have shape ", shape, ", not ", t.sizes());
}

inline void check_dense(const at::Tensor& t, const char* name) {
  TORCH_CHECK_VALUE(t.is_contiguous(), name, " must be contiguous");
  TORCH_CHECK_VALUE(reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0, name, " must be 16-byte aligned");
}

inline double number(PyObject* o, const char* name) {
  const double x = PyFloat_AsDouble(o);
  if (x == -1.0 && PyErr_Occurred()) {
    PyErr_Clear();
    TORCH_CHECK_TYPE(false, name, " must be a number");
  }
  return x;
}

inline int64_t whole(PyObject* o, const char* name) {
  const long long x = PyLong_AsLongLong(o);
  if (x == -1 && PyErr_Occurred()) {
    PyErr_Clear();
    TORCH_CHECK_TYPE(false, name, " must be a whole number of 64 bits");
  }
  return x;
}

inline bool truth(PyObject* o, const char* name) {
  const int x = PyObject_IsTrue(o);
  if (x < 0) {
    PyErr_Clear();
    TORCH_CHECK_TYPE(false, name, " must be a truth value");
  }
  return x != 0;
}

// Strides {sequence, row, head} of [batch, rows, heads, d] or, without a first
// axis, [rows, heads, d]; those of axes with one entry do not matter.
inline void strides_of(const at::Tensor& t, const char* name, int64_t (&s)[3]) {
  const int64_t per = 16 / t.element_size(), n = t.dim();
  bool fits = reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0 && (t.size(n - 1) <= 1 || t.stride(n - 1) == 1);
  for (int i = 0; i < 3; ++i) {
    const int64_t axis = n - 4 + i;
    s[i] = axis < 0 || t.size(axis) <= 1 ? 0 : t.stride(axis);
    fits = fits && s[i] % per == 0 && s[i] >= 0;
  }
  TORCH_CHECK_VALUE(fits || t.numel() == 0, name, " must have contiguous rows that start at multiples of 16 bytes");
}

template <class... T>
PyObject* tuple_of(const T&... t) {
  THPObjectPtr items[] = {THPObjectPtr(THPVariable_Wrap(t))...};
  for (const auto& i : items)
    if (!i) return nullptr;
  PyObject* r = PyTuple_New(sizeof...(t));
  if (r)
    for (size_t i = 0; i < sizeof...(t); ++i) PyTuple_SET_ITEM(r, i, items[i].release());
  return r;
}

inline at::Tensor bytes(int64_t n, const at::Tensor& ref) {
  return n > 0 ? at::empty({n}, at::TensorOptions().dtype(at::kByte).device(ref.device())) : at::Tensor();
}
inline void* pointer(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }

// A tensor that a kernel writes to, as an operation in place marks it.
inline void changed(const at::Tensor& t) {
  if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}

template <PyObject* (*F)(PyObject*, PyObject* const*, Py_ssize_t)>
PyMethodDef method(const char* name) {
  return {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(F)), METH_FASTCALL, nullptr};
}

}  // namespace binding
