// The binding's calls that take tensors as they come, over torch's C++ tensors:
// in Python a gradient set of hundreds of tensors costs 0.4 us a tensor, and a
// router call 6 us around its launch, more than their kernels take.
//
//   pack(grads, outs) -> (table, device)
//     table: bytes, a topoep_grad for each tensor (outs None: the gradients
//     themselves); device: the index of the GPU that all of them are on.
//   written(tensors): raises their version counters, so that autograd refuses a
//     backward pass that saved one of them before.
//   route(entry, router, logits, bias, stream) -> (code, ids, weights)
//   route_backward(entry, router, logits, ids, grad_weights, stream) -> (code, grad_logits)
//   moe_few(entry, router, x, gate, up, down, bias, expert_slot, workspace, stream) -> (code, out, ids, weights)
//     entry: the address of topoep_route (topoep_route_backward, topoep_moe_few);
//     router: of a topoep_router, whose dtype is the logits'; code: what it returned.
//
// TypeError and ValueError for what the library does not take, RuntimeError for
// tensors of forward-mode differentiation, whose tangents would be lost.  C++
// exceptions become what torch raises for them (memory that does not suffice:
// torch.OutOfMemoryError).
#include "tensors.h"

#include "topoep_moe.h"

namespace {

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
  THPObjectPtr table(PyBytes_FromStringAndSize(nullptr, n * (Py_ssize_t)sizeof(topoep_grad)));
  if (!table) return nullptr;
  topoep_grad *to = reinterpret_cast<topoep_grad *>(PyBytes_AS_STRING(table.get()));
  int device = -1;
  const bool tangents = any_tangents();
  for (Py_ssize_t i = 0; i < n; ++i) {
    PyObject *pg = PySequence_Fast_GET_ITEM(grads, i), *po = outs ? PySequence_Fast_GET_ITEM(outs, i) : pg;
    if (!THPVariable_Check(pg) || !THPVariable_Check(po)) return refuse(PyExc_TypeError, "not a tensor", i);
    const at::Tensor &g = THPVariable_Unpack(pg), &o = THPVariable_Unpack(po);
    if (tangents && (has_tangent(g) || has_tangent(o))) return refuse(PyExc_RuntimeError, "carries a tangent, which is not passed on", i);
    if (!g.is_cuda() || !o.is_cuda()) return refuse(PyExc_ValueError, "not on a GPU", i);
    if (g.layout() != at::kStrided || o.layout() != at::kStrided) return refuse(PyExc_TypeError, "not a strided tensor", i);
    if (device < 0) device = g.get_device();
    if (g.get_device() != device || o.get_device() != device) return refuse(PyExc_ValueError, "on another GPU than the first", i);
    const int from = dtype_of(g), into = dtype_of(o);
    if (from < 0 || into < 0) return refuse(PyExc_TypeError, "not float32, bfloat16 or float16", i);
    if (po != pg && !g.sizes().equals(o.sizes())) return refuse(PyExc_ValueError, "its output has another shape", i);
    if (!(g.is_contiguous() && o.is_contiguous()) &&
        !(g.is_non_overlapping_and_dense() && g.strides().equals(o.strides())))
      return refuse(PyExc_ValueError, "not dense, or its output has other strides", i);
    to[i].grad = g.data_ptr();
    to[i].out = o.data_ptr();
    to[i].n = g.numel();
    to[i].dtype = from;
    to[i].out_dtype = into;
  }
  return Py_BuildValue("(Ni)", table.release(), device);
}

PyObject *pack(PyObject *, PyObject *args) {
  PyObject *grads = nullptr, *outs = nullptr;
  if (!PyArg_ParseTuple(args, "OO", &grads, &outs)) return nullptr;
  THPObjectPtr fg(PySequence_Fast(grads, "grads is a list of tensors")), fo;
  if (!fg) return nullptr;
  if (outs != Py_None) {
    fo = PySequence_Fast(outs, "outs is a list of tensors");
    if (!fo) return nullptr;
  }
  return guarded([&] { return fill(fg.get(), fo.get()); });
}

PyObject *written(PyObject *, PyObject *tensors) {
  PyObject *fast = PySequence_Fast(tensors, "a list of tensors");
  if (!fast) return nullptr;
  for (Py_ssize_t i = 0; i < PySequence_Fast_GET_SIZE(fast); ++i) {
    const at::Tensor &t = THPVariable_Unpack(PySequence_Fast_GET_ITEM(fast, i));   // pack() took it
    if (!t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
  }
  Py_DECREF(fast);
  Py_RETURN_NONE;
}

PyObject *route(PyObject *, PyObject *args) {
  unsigned long long entry, router, stream;
  PyObject *pl, *pb;
  if (!PyArg_ParseTuple(args, "KKOOK", &entry, &router, &pl, &pb, &stream)) return nullptr;
  return guarded([&]() -> PyObject * {
    const topoep_router *r = reinterpret_cast<const topoep_router *>(router);
    const at::Tensor *x = tensor_of(pl, "logits"), *b = pb == Py_None ? nullptr : tensor_of(pb, "bias");
    if (!x || (pb != Py_None && !b)) return nullptr;
    const int64_t ld = row_stride(*x, "logits");
    if (ld < 0 || (b && !dense(*b, "bias", at::kFloat, *x, {x->size(1)}))) return nullptr;
    const at::TensorOptions on = x->options();
    at::Tensor ids = at::empty({x->size(0), r->topk}, on.dtype(at::kInt));
    at::Tensor weights = at::empty({x->size(0), r->topk}, on.dtype(at::kFloat));
    const int rc = x->size(0) > INT32_MAX ? TOPOEP_EINVAL
                                          : reinterpret_cast<decltype(&topoep_route)>(entry)(
                                                r, x->data_ptr(), ld, (int32_t)x->size(0), b ? b->data_ptr<float>() : nullptr,
                                                ids.data_ptr<int32_t>(), weights.data_ptr<float>(),
                                                reinterpret_cast<void *>(stream));
    return Py_BuildValue("(iNN)", rc, THPVariable_Wrap(ids), THPVariable_Wrap(weights));
  });
}

PyObject *route_backward(PyObject *, PyObject *args) {
  unsigned long long entry, router, stream;
  PyObject *pl, *pi, *pg;
  if (!PyArg_ParseTuple(args, "KKOOOK", &entry, &router, &pl, &pi, &pg, &stream)) return nullptr;
  return guarded([&]() -> PyObject * {
    const topoep_router *r = reinterpret_cast<const topoep_router *>(router);
    const at::Tensor *x = tensor_of(pl, "logits"), *ids = tensor_of(pi, "ids"), *g = tensor_of(pg, "grad_weights");
    if (!x || !ids || !g) return nullptr;
    const int64_t ld = row_stride(*x, "logits");
    if (ld < 0 || !dense(*ids, "ids", at::kInt, *x, {x->size(0), r->topk}) ||
        !dense(*g, "grad_weights", at::kFloat, *x, {x->size(0), r->topk}))
      return nullptr;
    at::Tensor out = at::empty({x->size(0), x->size(1)}, x->options());
    const int rc = x->size(0) > INT32_MAX
                       ? TOPOEP_EINVAL
                       : reinterpret_cast<decltype(&topoep_route_backward)>(entry)(
                             r, x->data_ptr(), ld, (int32_t)x->size(0), ids->data_ptr<int32_t>(), g->data_ptr<float>(),
                             out.data_ptr(), x->size(1), reinterpret_cast<void *>(stream));
    return Py_BuildValue("(iN)", rc, THPVariable_Wrap(out));
  });
}

PyObject *moe_few(PyObject *, PyObject *args) {
  unsigned long long entry, router, stream;
  PyObject *px, *pg, *pu, *pd, *pb, *ps, *pw;
  if (!PyArg_ParseTuple(args, "KKOOOOOOOK", &entry, &router, &px, &pg, &pu, &pd, &pb, &ps, &pw, &stream)) return nullptr;
  return guarded([&]() -> PyObject * {
    const topoep_router *r = reinterpret_cast<const topoep_router *>(router);
    const at::Tensor *x = tensor_of(px, "x"), *gate = tensor_of(pg, "gate"), *up = tensor_of(pu, "up"),
                     *down = tensor_of(pd, "down"), *ws = tensor_of(pw, "workspace");
    if (!x || !gate || !up || !down || !ws) return nullptr;
    const at::Tensor *bias = pb == Py_None ? nullptr : tensor_of(pb, "bias");
    const at::Tensor *slot = ps == Py_None ? nullptr : tensor_of(ps, "expert_slot");
    if ((pb != Py_None && !bias) || (ps != Py_None && !slot)) return nullptr;
    const int64_t ldx = row_stride(*x, "x");
    if (ldx < 0) return nullptr;
    const at::ScalarType type = x->scalar_type();
    if (type != at::kBFloat16 && type != at::kHalf) {
      PyErr_SetString(PyExc_TypeError, "x must be bfloat16 or float16");
      return nullptr;
    }
    if (gate->dim() != 2 || up->dim() != 3 || down->dim() != 3) {
      PyErr_SetString(PyExc_ValueError, "gate is [E, H], up [L, 2I, H], down [L, H, I]");
      return nullptr;
    }
    const int64_t T = x->size(0), H = x->size(1), E = gate->size(0), L = down->size(0), I = down->size(2);
    if (!dense(*gate, "gate", type, *x, {E, H}) || !dense(*up, "up", type, *x, {L, 2 * I, H}) ||
        !dense(*down, "down", type, *x, {L, H, I}) || (bias && !dense(*bias, "bias", at::kFloat, *x, {E})) ||
        (slot && !dense(*slot, "expert_slot", at::kInt, *x, {E})))
      return nullptr;
    if (ws->device() != x->device() || !ws->is_contiguous()) {
      PyErr_SetString(PyExc_ValueError, "workspace must be contiguous on the same GPU");
      return nullptr;
    }
    const uintptr_t from = reinterpret_cast<uintptr_t>(ws->data_ptr()), at = (from + 255) & ~(uintptr_t)255;
    const size_t size = ws->nbytes() > at - from ? ws->nbytes() - (at - from) : 0;
    at::Tensor out = at::empty({T, H}, x->options());
    at::Tensor ids = at::empty({T, r->topk}, x->options().dtype(at::kInt));
    at::Tensor weights = at::empty({T, r->topk}, x->options().dtype(at::kFloat));
    const auto fits = [](int64_t v) { return v <= INT32_MAX; };
    const topoep_moe m{(int32_t)H, (int32_t)I, (int32_t)L, type == at::kHalf ? TOPOEP_F16 : TOPOEP_BF16};
    const int rc = !fits(T) || !fits(H) || !fits(I) || !fits(L)
                       ? TOPOEP_EINVAL
                       : reinterpret_cast<decltype(&topoep_moe_few)>(entry)(
                             &m, r, x->data_ptr(), ldx, (int32_t)T, gate->data_ptr(), bias ? bias->data_ptr<float>() : nullptr,
                             slot ? slot->data_ptr<int32_t>() : nullptr, up->data_ptr(), down->data_ptr(), out.data_ptr(),
                             ids.data_ptr<int32_t>(), weights.data_ptr<float>(), reinterpret_cast<void *>(at), size,
                             reinterpret_cast<void *>(stream));
    return Py_BuildValue("(iNNN)", rc, THPVariable_Wrap(out), THPVariable_Wrap(ids), THPVariable_Wrap(weights));
  });
}

PyMethodDef methods[] = {{"moe_few", moe_few, METH_VARARGS,
                          "moe_few(entry, router, x, gate, up, down, bias, expert_slot, workspace, stream) -> (code, out, ids, weights)"},
                         {"route", route, METH_VARARGS, "route(entry, router, logits, bias, stream) -> (code, ids, weights)"},
                         {"route_backward", route_backward, METH_VARARGS,
                          "route_backward(entry, router, logits, ids, grad_weights, stream) -> (code, grad_logits)"},
                         {"pack", pack, METH_VARARGS, "pack(grads, outs) -> (bytes, device)"},
                         {"written", written, METH_O, "written(tensors)"}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__tensors() { return PyModule_Create(&module); }
