// binding.h -- what the calls on torch tensors share: which tensors they take.
#pragma once

#include <torch/csrc/jit/frontend/tracer.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <c10/core/impl/LocalDispatchKeySet.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include "fewbit.h"

namespace binding {

// Storage type of the C ABI, or -1.
inline int storage_type(const at::Tensor& t) {
  switch (t.scalar_type()) {
    case at::kFloat: return FEWBIT_F32;
    case at::kHalf: return FEWBIT_F16;
    case at::kBFloat16: return FEWBIT_BF16;
    default: return -1;
  }
}

// Nothing watches or rewrites tensor operations on this thread.
inline bool plain_mode() {
  return !c10::impl::TorchDispatchModeTLS::any_modes_set() && !at::impl::torch_function_mode_enabled() &&
         !torch::jit::tracer::isTracing() &&
         !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::FuncTorchDynamicLayerFrontMode) &&
         !c10::impl::tls_is_dispatch_key_included(c10::DispatchKey::PythonTLSSnapshot);
}

// An ordinary dense device tensor, not a wrapper and not a lazy view.
inline bool plain(const at::Tensor& t) {
  constexpr c10::DispatchKeySet kOdd({c10::DispatchKey::Python, c10::DispatchKey::FuncTorchGradWrapper,
                                      c10::DispatchKey::FuncTorchBatched, c10::DispatchKey::Functionalize,
                                      c10::DispatchKey::ZeroTensor, c10::DispatchKey::Conjugate,
                                      c10::DispatchKey::Negative});
  return t.is_cuda() && t.layout() == at::kStrided && !t.key_set().has_any(kOdd);
}

inline void* stream_of(const at::Tensor& t) {
  return c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(t.device().index()).stream();
}

// The block operators' calls (binding_block.cpp).
PyMethodDef* block_methods();

}  // namespace binding
