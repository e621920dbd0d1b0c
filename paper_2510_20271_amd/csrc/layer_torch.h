// What the autograd functions in C++ share: errors, the current stream, checks of tensors.
#pragma once
#include <torch/extension.h>

#include <c10/hip/HIPStream.h>

#include <string>

#include "ecc.h"

void bind_operators(py::module_& m);  // operators_torch.cpp

namespace {

using torch::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

// What the library refuses is the Python binding's EccError, with its status, in the backward pass as well.
inline void check(int status) {
  if (status == ECC_OK) return;
  const std::string message = ecc_last_error();  // (of this thread)
  const py::gil_scoped_acquire gil;
  const py::object type = py::module_::import("paper_2510_20271_amd.api").attr("EccError");
  const py::object error = type(status, message);
  PyErr_SetObject(type.ptr(), error.ptr());
  throw py::error_already_set();
}
inline void* stream() { return c10::hip::getCurrentHIPStream().stream(); }
inline float* f32(const Tensor& t) { return t.defined() ? t.data_ptr<float>() : nullptr; }
// Saved tensors come back from saved-tensor hooks, upstream gradients from anywhere: what the kernels are handed is as the
// forward pass made it, or nothing (numel < 0: any number of elements).
inline void check_device(const Tensor& t, at::ScalarType type, int64_t numel, const at::Device& device) {
  TORCH_CHECK_VALUE(t.defined() && t.layout() == at::kStrided && t.has_storage() && t.is_contiguous() && t.device() == device,
                    "tensors must be contiguous device tensors");
  TORCH_CHECK_VALUE(t.scalar_type() == type && (numel < 0 || t.numel() == numel),
                    "a saved tensor or gradient is not of the type or size that the forward pass left");
}

}  // namespace
