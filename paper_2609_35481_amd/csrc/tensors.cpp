// Reads lists of torch tensors for the binding: a gradient set of hundreds of
// tensors costs some 0.4 us a tensor in Python, more than its kernels take.
//
//   pack(grads, outs) -> (table, device)
//
// table: bytes, a topoep_grad for each tensor (outs None: the gradients
// themselves); device: the index of the GPU that all of them are on.  Raises
// TypeError and ValueError for what the library does not take.
#define PY_SSIZE_T_CLEAN
#include <torch/csrc/autograd/python_variable.h>

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

PyObject *refuse(PyObject *kind, const char *what, Py_ssize_t i) {
  PyErr_Format(kind, "tensor %zd: %s", i, what);
  return nullptr;
}

PyObject *fill(PyObject *grads, PyObject *outs) {
  const Py_ssize_t n = PySequence_Fast_GET_SIZE(grads);
  if (outs && PySequence_Fast_GET_SIZE(outs) != n) {
    PyErr_Format(PyExc_ValueError, "%zd outs for %zd grads", PySequence_Fast_GET_SIZE(outs), n);
    return nullptr;
  }
  PyObject *table = PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(topoep_grad));
  if (!table) return nullptr;
  topoep_grad *to = reinterpret_cast<topoep_grad *>(PyBytes_AS_STRING(table));
  int device = -1;
  const auto drop = [&](PyObject *kind, const char *what, Py_ssize_t i) {
    Py_DECREF(table);
    return refuse(kind, what, i);
  };
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *pg = PySequence_Fast_GET_ITEM(grads, i), *po = outs ? PySequence_Fast_GET_ITEM(outs, i) : pg;
    if (!THPVariable_Check(pg) || !THPVariable_Check(po)) return drop(PyExc_TypeError, "not a tensor", i);
    const at::Tensor &g = THPVariable_Unpack(pg), &o = THPVariable_Unpack(po);
    if (!g.is_cuda() || !o.is_cuda()) return drop(PyExc_ValueError, "not on a GPU", i);
    if (g.layout() != at::kStrided || o.layout() != at::kStrided) return drop(PyExc_TypeError, "not a strided tensor", i);
    if (device < 0) device = g.get_device();
    if (g.get_device() != device || o.get_device() != device) return drop(PyExc_ValueError, "on another GPU than the first", i);
    const int from = dtype_of(g), into = dtype_of(o);
    if (from < 0 || into < 0) return drop(PyExc_TypeError, "not float32, bfloat16 or float16", i);
    if (po != pg && !g.sizes().equals(o.sizes())) return drop(PyExc_ValueError, "its output has another shape", i);
    if (!(g.is_contiguous() && o.is_contiguous()) &&
        !(g.is_non_overlapping_and_dense() && g.strides().equals(o.strides())))
      return drop(PyExc_ValueError, "not dense, or its output has other strides", i);
    to[i].grad = g.data_ptr();
    to[i].out = o.data_ptr();
    to[i].n = g.numel();
    to[i].dtype = from;
    to[i].out_dtype = into;
  }
  PyObject *both = Py_BuildValue("(Ni)", table, device);
  return both;
}

PyObject *pack(PyObject *, PyObject *args) {
  PyObject *grads = nullptr, *outs = nullptr;
  if (!PyArg_ParseTuple(args, "OO", &grads, &outs)) return nullptr;
  PyObject *fg = PySequence_Fast(grads, "grads is a list of tensors");
  if (!fg) return nullptr;
  PyObject *fo = nullptr;
  if (outs != Py_None) {
    fo = PySequence_Fast(outs, "outs is a list of tensors");
    if (!fo) {
      Py_DECREF(fg);
      return nullptr;
    }
  }
  PyObject *result = nullptr;
  try {
    result = fill(fg, fo);
  } catch (const std::exception &e) {
    PyErr_SetString(PyExc_RuntimeError, e.what());
  }
  Py_DECREF(fg);
  Py_XDECREF(fo);
  return result;
}

PyMethodDef methods[] = {{"pack", pack, METH_VARARGS, "pack(grads, outs) -> (bytes, device)"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
