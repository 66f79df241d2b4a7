// What the binding's modules over torch's C++ tensors share: checks of arguments, whose
// errors are TypeError, ValueError and RuntimeError (tangents), and C++ exceptions as torch's own.
#pragma once

#define PY_SSIZE_T_CLEAN
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/forward_grad.h>
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/object_ptr.h>

#include <ATen/ops/empty.h>
#include <Python.h>

#include "topoep_moe.h"

namespace {

int dtype_of(const at::Tensor &t) {
  switch (t.scalar_type()) {
    case at::kFloat: return TOPOEP_F32;
    case at::kBFloat16: return TOPOEP_BF16;
    case at::kHalf: return TOPOEP_F16;
    default: return -1;
  }
}

// Whether tangents exist at all: asking each tensor takes 35 ns, a view's base among them.
bool any_tangents() { return torch::autograd::ForwardADLevel::try_get_by_idx(0) != nullptr; }
bool has_tangent(const at::Tensor &t) { return t._fw_grad(0).defined(); }

template <class F>
PyObject *guarded(const F &f) {
  try {
    return f();
  } catch (...) {
    torch::translate_exception_to_python(std::current_exception());
    return nullptr;
  }
}

// Row stride of a matrix of dense rows that do not overlap; -1 (and an error)
// for anything else.
int64_t row_stride(const at::Tensor &t, const char *name) {
  if (!t.is_cuda()) {
    PyErr_Format(PyExc_TypeError, "%s must be a CUDA tensor", name);
    return -1;
  }
  if (t.dim() != 2 || (t.size(1) > 1 && t.stride(1) != 1) || (t.size(0) > 1 && t.stride(0) < t.size(1))) {
    PyErr_Format(PyExc_ValueError, "%s must be a matrix of dense rows that do not overlap", name);
    return -1;
  }
  return t.size(0) > 1 ? t.stride(0) : t.size(1);
}

bool dense(const at::Tensor &t, const char *name, at::ScalarType type, const at::Tensor &like, at::IntArrayRef shape) {
  if (t.scalar_type() != type || t.device() != like.device()) {
    PyErr_Format(PyExc_TypeError, "%s must be %s on the same GPU", name, c10::toString(type));
    return false;
  }
  if (!t.sizes().equals(shape) || !t.is_contiguous()) {
    PyErr_Format(PyExc_ValueError, "%s must be contiguous and of the shape that goes with the others", name);
    return false;
  }
  return true;
}

const at::Tensor *tensor_of(PyObject *o, const char *name) {
  if (!THPVariable_Check(o)) {
    PyErr_Format(PyExc_TypeError, "%s is not a tensor", name);
    return nullptr;
  }
  const at::Tensor &t = THPVariable_Unpack(o);
  if (!any_tangents() || !has_tangent(t)) return &t;
  PyErr_Format(PyExc_RuntimeError, "%s carries a tangent, which is not passed on", name);
  return nullptr;
}

}  // namespace
