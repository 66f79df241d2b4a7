// The binding's calls of the experts' products over torch's C++ tensors: a routed
// layer's training step is a dozen kernels, around which checks, allocations
// and autograd take longer in Python than small layers' kernels do.
//
//   bind(addresses): of the library's entries, in the order of Entries
//   expert_rows(ids, L, slot, stream) -> (code, offsets, pairs, places)
//   block(x, ids, weights, up, down, slot, stream) -> (code, out)
//     ids, weights and slot None: the dense block
//   quantize(x, stream) -> (code, q, scale)
//   matmul_int8(x, scale, w, w_scale, offsets, gated, type, out, stream) -> (code, out)
//     scale None: x is quantised first; type: of a new out, -1 for x's; out: None or where to
//
// code: what the library returned; with one other than TOPOEP_OK the rest is None.
#include "tensors.h"

#include <ATen/core/grad_mode.h>
#include <ATen/hip/impl/HIPStreamMasqueradingAsCUDA.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/autograd/functions/basic_ops.h>

#include "topoep_ffn.h"

namespace {

using at::Tensor;
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

struct Entries {
  decltype(&topoep_expert_rows_workspace_bytes) rows_bytes;
  decltype(&topoep_expert_rows) rows;
  decltype(&topoep_ffn_bytes) bytes;
  decltype(&topoep_ffn_forward) forward;
  decltype(&topoep_ffn_backward) backward;
  decltype(&topoep_quantize) quantize;
  decltype(&topoep_matmul_int8_workspace_bytes) int8_bytes;
  decltype(&topoep_matmul_int8) int8;
} entry;

struct Code { int rc; };                                  // thrown: what the library returned
void check(int rc) { if (rc != TOPOEP_OK) throw Code{rc}; }
struct Refused {};                                        // thrown: a Python error is set

[[noreturn]] void refuse(PyObject *kind, const char *what) {
  PyErr_SetString(kind, what);
  throw Refused();
}
int32_t fits(int64_t v) { return v <= INT32_MAX ? (int32_t)v : throw Code{TOPOEP_EINVAL}; }

// A tensor of `dims` dimensions.
const Tensor &given(PyObject *o, const char *name, int64_t dims) {
  const Tensor *t = tensor_of(o, name);
  if (!t) throw Refused();
  if (t->dim() != dims) {
    PyErr_Format(PyExc_ValueError, "%s must have %lld dimensions, not %lld", name, (long long)dims, (long long)t->dim());
    throw Refused();
  }
  return *t;
}
const Tensor &on_gpu(const Tensor &t, const char *name) {
  if (!t.is_cuda()) {
    PyErr_Format(PyExc_TypeError, "%s must be on a GPU", name);
    throw Refused();
  }
  return t;
}
int64_t stride_of(const Tensor &t, const char *name) {
  const int64_t ld = row_stride(t, name);
  if (ld < 0) throw Refused();
  return t.size(0) > 1 ? ld : (ld + 15) / 16 * 16;        // (of one row anything)
}
void is_dense(const Tensor &t, const char *name, at::ScalarType type, const Tensor &like, at::IntArrayRef shape) {
  if (!dense(t, name, type, like, shape)) throw Refused();
}

Tensor scratch(size_t n, const Tensor &like) { return at::empty({(int64_t)(n ? n : 1)}, like.options().dtype(at::kByte)); }
void *at_of(const Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

template <class F>
PyObject *answered(const F &f) {
  return guarded([&]() -> PyObject * {
    try {
      return f();
    } catch (const Code &c) {
      return Py_BuildValue("(iOOO)", c.rc, Py_None, Py_None, Py_None);
    } catch (const Refused &) {
      return nullptr;
    }
  });
}

// ---------------------------------------------------------------- rows by expert

struct Rows { Tensor offsets, pairs, places; };

Rows rows_of(const Tensor &ids, int32_t L, const Tensor &slot, void *stream) {
  const int32_t T = fits(ids.size(0)), k = fits(ids.size(1));
  on_gpu(ids, "ids");
  is_dense(ids, "ids", at::kInt, ids, {T, k});
  const int32_t E = slot.defined() ? fits(slot.size(0)) : L;
  if (slot.defined()) is_dense(slot, "expert_slot", at::kInt, ids, {E});
  size_t need = 0;
  check(entry.rows_bytes(T, k, L, &need));
  Rows r{at::empty({(int64_t)L + 1}, ids.options()), at::empty({(int64_t)T * k}, ids.options()), at::empty({T, k}, ids.options())};
  const Tensor ws = scratch(need, ids);
  check(entry.rows(ids.data_ptr<int32_t>(), T, k, slot.defined() ? slot.data_ptr<int32_t>() : nullptr, E, L,
                   r.offsets.data_ptr<int32_t>(), r.pairs.data_ptr<int32_t>(), r.places.data_ptr<int32_t>(), ws.data_ptr(),
                   (size_t)ws.numel(), stream));
  return r;
}

// ---------------------------------------------------------------- the gated block

// A call's operands as the library takes them.
struct Block {
  topoep_ffn f;
  topoep_ffn_rows r;
  const topoep_ffn_rows *rows;
  int32_t T;
  int64_t ldx;
  size_t forward, saved, backward;
  Block(const Tensor &x, int64_t stride, const Tensor &weights, const Tensor &up, const Tensor &down, const Rows &by, int64_t E) {
    const bool routed = weights.defined();
    f = topoep_ffn{fits(down.size(-2)), fits(down.size(-1)), routed ? fits(up.size(0)) : 1, dtype_of(x)};
    T = fits(x.size(0));
    ldx = stride;
    rows = routed ? &r : nullptr;
    if (routed)
      r = topoep_ffn_rows{by.offsets.data_ptr<int32_t>(), by.pairs.data_ptr<int32_t>(), by.places.data_ptr<int32_t>(),
                          weights.data_ptr<float>(), fits(weights.size(1)), fits(E)};
    check(entry.bytes(&f, T, rows, &forward, &saved, &backward));
  }
};

Tensor forward(const Tensor &x, const Tensor &weights, const Tensor &up, const Tensor &down, const Rows &by, int64_t E,
               Tensor *saved, void *stream) {
  const Block b(x, stride_of(x, "x"), weights, up, down, by, E);
  Tensor out = at::empty(x.sizes(), x.options());
  if (saved) *saved = scratch(b.saved, x);
  const Tensor ws = scratch(b.forward, x);
  check(entry.forward(&b.f, x.data_ptr(), b.ldx, b.T, b.rows, up.data_ptr(), down.data_ptr(), out.data_ptr(),
                      saved ? saved->data_ptr() : nullptr, ws.data_ptr(), (size_t)ws.numel(), stream));
  return out;
}

// What a hook on saved tensors gave back for one of them.  It keeps the value, shape and type of what was saved, and the
// GPU, but not its layout; the kernels read dense tensors at multiples of 16 bytes.  (No Python here: a backward pass does
// not hold its lock.)
void is_alike(const Tensor &t, const char *name, at::ScalarType type, const Tensor &like, at::IntArrayRef shape) {
  TORCH_CHECK(t.defined() && t.layout() == at::kStrided && t.scalar_type() == type && t.device() == like.device() &&
                  t.sizes().equals(shape),
              "a hook on saved tensors gave back another ", name, " than was saved: it has to be ", type, " of shape ", shape, " on ", like.device());
}
bool aligned(const Tensor &t) { return reinterpret_cast<uintptr_t>(t.data_ptr()) % 16 == 0; }
Tensor at_16(const Tensor &t) { return aligned(t) ? t : t.clone(); }
Tensor given_back(const Tensor &t, const char *name, at::ScalarType type, const Tensor &like, at::IntArrayRef shape) {
  is_alike(t, name, type, like, shape);
  return at_16(t.contiguous());
}

struct FeedForward : torch::autograd::Function<FeedForward> {
  static Tensor forward(AutogradContext *ctx, const Tensor &x, const std::optional<Tensor> &routers, const Tensor &up,
                        const Tensor &down, const Rows &by, int64_t E, int64_t stream) {
    const Tensor weights = routers.value_or(Tensor());
    Tensor saved;
    const Tensor out = ::forward(x, weights, up, down, by, E, &saved, reinterpret_cast<void *>(stream));
    ctx->save_for_backward({x, weights, up, down, saved});
    ctx->saved_data["E"] = E;
    ctx->saved_data["I"] = down.size(-1);
    if (weights.defined()) {   // out of a hook's reach: kernels read at what these name
      ctx->saved_data["offsets"] = by.offsets;
      ctx->saved_data["pairs"] = by.pairs;
      ctx->saved_data["places"] = by.places;
    }
    return out;
  }
  static variable_list backward(AutogradContext *ctx, variable_list grads) {
    const variable_list s = ctx->get_saved_variables();
    variable_list out(7);
    int rc = TOPOEP_OK;
    {
      at::AutoGradMode off(false);
      const Tensor grad = at_16(grads[0].contiguous());   // [T, H]: autograd sees to that
      const bool routed = ctx->saved_data.count("offsets") > 0;
      const at::ScalarType type = grad.scalar_type();
      const int64_t T = grad.size(0), H = grad.size(1);
      Tensor weights;
      Rows by;
      std::vector<int64_t> shape;                         // of the experts, if there are any
      if (routed) {
        by = Rows{ctx->saved_data["offsets"].toTensor(), ctx->saved_data["pairs"].toTensor(), ctx->saved_data["places"].toTensor()};
        weights = given_back(s[1], "weights", at::kFloat, grad, by.places.sizes());
        shape.push_back(by.offsets.size(0) - 1);
      }
      const int64_t I = ctx->saved_data["I"].toInt();
      const size_t n = shape.size();
      shape.insert(shape.end(), {2 * I, H});
      const Tensor up = given_back(s[2], "up", type, grad, shape);
      shape[n] = H, shape[n + 1] = I;
      const Tensor down = given_back(s[3], "down", type, grad, shape);
      is_alike(s[0], "x", type, grad, {T, H});
      const bool rows = s[0].stride(1) == 1 && (T < 2 || (s[0].stride(0) >= H && s[0].stride(0) % 8 == 0)) && aligned(s[0]);
      const Tensor x = rows ? s[0] : at_16(s[0].contiguous());
      try {
        const Block b(x, T > 1 ? x.stride(0) : H, weights, up, down, by, ctx->saved_data["E"].toInt());
        const Tensor saved = given_back(s[4], "block's values", at::kByte, grad, {(int64_t)(b.saved ? b.saved : 1)});
        size_t edge = 0;
        const Tensor *like[] = {&x, &weights, &up, &down};
        for (int i = 0; i < 4; ++i) {
          if (!like[i]->defined()) continue;   // (not an input then)
          if (ctx->needs_input_grad(edge++)) out[i] = at::empty(like[i]->sizes(), like[i]->options());
        }
        const Tensor ws = scratch(b.backward, x);
        void *stream = c10::hip::getCurrentHIPStreamMasqueradingAsCUDA(x.get_device()).stream();
        rc = entry.backward(&b.f, x.data_ptr(), b.ldx, b.T, b.rows, up.data_ptr(), down.data_ptr(), saved.data_ptr(),
                            grad.data_ptr(), at_of(out[0]), static_cast<float *>(at_of(out[1])), at_of(out[2]),
                            at_of(out[3]), ws.data_ptr(), (size_t)ws.numel(), stream);
      } catch (const Code &c) {
        rc = c.rc;
      }
      TORCH_CHECK(rc == TOPOEP_OK, "topoep_ffn_backward failed with code ", rc);
    }
    if (at::GradMode::is_enabled()) {                     // a gradient through the gradients is an error
      const auto error = std::make_shared<torch::autograd::DelayedError>("the gradients of the gated block have none of their own", 1);
      for (Tensor &t : out)
        if (t.defined()) {
          t = t.detach();
          t.set_requires_grad(true);
          t = (*error)({t})[0];
        }
    }
    return out;
  }
};

bool watched(std::initializer_list<const Tensor *> ts) {
  if (!at::GradMode::is_enabled()) return false;
  for (const Tensor *t : ts)
    if (t->defined() && t->requires_grad()) return true;
  return false;
}

// ---------------------------------------------------------------- 8-bit integers

void quantize(const Tensor &x, Tensor &q, Tensor &scale, void *stream) {
  on_gpu(x, "x");
  const int type = dtype_of(x);
  if (type < 0) refuse(PyExc_TypeError, "x must be float32, bfloat16 or float16");
  const int64_t ld = stride_of(x, "x");
  const int32_t M = fits(x.size(0)), K = fits(x.size(1));
  q = at::empty({M, K}, x.options().dtype(at::kChar));
  scale = at::empty({M}, x.options().dtype(at::kFloat));
  check(entry.quantize(x.data_ptr(), type, ld, M, K, q.data_ptr<int8_t>(), scale.data_ptr<float>(), stream));
}

// A result that has no gradient, where one is asked for: a backward pass through it is an error.
Tensor forward_only(const Tensor &t, const char *what) {
  const auto error = std::make_shared<torch::autograd::DelayedError>(what, 1);
  Tensor v = t.detach();
  v.set_requires_grad(true);
  return (*error)({v})[0];
}

// ---------------------------------------------------------------- Python

PyObject *bind(PyObject *, PyObject *args) {
  unsigned long long a[8];
  if (!PyArg_ParseTuple(args, "KKKKKKKK", a, a + 1, a + 2, a + 3, a + 4, a + 5, a + 6, a + 7)) return nullptr;
  static_assert(sizeof(Entries) == sizeof(a), "eight addresses");
  memcpy(&entry, a, sizeof(a));
  Py_RETURN_NONE;
}

Tensor optional(PyObject *o, const char *name, int64_t dims) { return o == Py_None ? Tensor() : given(o, name, dims); }

PyObject *expert_rows(PyObject *, PyObject *args) {
  unsigned long long stream;
  int L;
  PyObject *pi, *ps;
  if (!PyArg_ParseTuple(args, "OiOK", &pi, &L, &ps, &stream)) return nullptr;
  return answered([&] {
    const Rows r = rows_of(given(pi, "ids", 2), L, optional(ps, "expert_slot", 1), reinterpret_cast<void *>(stream));
    return Py_BuildValue("(iNNN)", TOPOEP_OK, THPVariable_Wrap(r.offsets), THPVariable_Wrap(r.pairs), THPVariable_Wrap(r.places));
  });
}

PyObject *block(PyObject *, PyObject *args) {
  unsigned long long stream;
  PyObject *px, *pi, *pw, *pu, *pd, *ps;
  if (!PyArg_ParseTuple(args, "OOOOOOK", &px, &pi, &pw, &pu, &pd, &ps, &stream)) return nullptr;
  return answered([&] {
    const bool routed = pi != Py_None;
    const int64_t dims = routed ? 3 : 2;
    const Tensor &x = on_gpu(given(px, "x", 2), "x"), &up = given(pu, "up", dims), &down = given(pd, "down", dims);
    if (x.scalar_type() != at::kBFloat16 && x.scalar_type() != at::kHalf)
      refuse(PyExc_TypeError, "x must be bfloat16 or float16");
    const int64_t L = routed ? up.size(0) : 1, H = down.size(-2), I = down.size(-1);
    if (x.size(1) != H) refuse(PyExc_ValueError, "x is [T, H], up [.., 2I, H], down [.., H, I]");
    if (routed) {
      is_dense(up, "up", x.scalar_type(), x, {L, 2 * I, H});
      is_dense(down, "down", x.scalar_type(), x, {L, H, I});
    } else {
      is_dense(up, "up", x.scalar_type(), x, {2 * I, H});
      is_dense(down, "down", x.scalar_type(), x, {H, I});
    }
    Tensor weights;
    Rows by;
    int64_t E = 1;
    if (routed) {
      const Tensor &ids = given(pi, "ids", 2);
      if (ids.size(0) != x.size(0) || ids.device() != x.device())
        refuse(PyExc_ValueError, "ids must have a row for each of x, on its GPU");
      const Tensor slot = optional(ps, "expert_slot", 1);
      weights = given(pw, "weights", 2);
      is_dense(weights, "weights", at::kFloat, x, ids.sizes());
      E = std::max<int64_t>(1, slot.defined() ? slot.size(0) : L);
      by = rows_of(ids, fits(L), slot, reinterpret_cast<void *>(stream));
    }
    Tensor out;
    if (watched({&x, &weights, &up, &down})) out = FeedForward::apply(x, routed ? std::optional<Tensor>(weights) : std::nullopt, up, down, by, E, (int64_t)stream);
    else out = forward(x, weights, up, down, by, E, nullptr, reinterpret_cast<void *>(stream));
    return Py_BuildValue("(iN)", TOPOEP_OK, THPVariable_Wrap(out));
  });
}

PyObject *quantize(PyObject *, PyObject *args) {
  unsigned long long stream;
  PyObject *px;
  if (!PyArg_ParseTuple(args, "OK", &px, &stream)) return nullptr;
  return answered([&] {
    const Tensor &x = given(px, "x", 2);
    Tensor q, scale;
    quantize(x, q, scale, reinterpret_cast<void *>(stream));
    if (watched({&x})) scale = forward_only(scale, "quantize is forward only: its inputs get no gradient");
    return Py_BuildValue("(iNN)", TOPOEP_OK, THPVariable_Wrap(q), THPVariable_Wrap(scale));
  });
}

PyObject *matmul_int8(PyObject *, PyObject *args) {
  unsigned long long stream;
  int gated, type;
  PyObject *px, *ps, *pw, *pws, *po, *pout;
  if (!PyArg_ParseTuple(args, "OOOOOpiOK", &px, &ps, &pw, &pws, &po, &gated, &type, &pout, &stream)) return nullptr;
  return answered([&] {
    void *const st = reinterpret_cast<void *>(stream);
    const Tensor &x = on_gpu(given(px, "x", 2), "x"), offsets = optional(po, "offsets", 1);
    const Tensor &w = given(pw, "w", offsets.defined() ? 3 : 2), &ws = given(pws, "w_scale", w.dim() - 1);
    Tensor scale = optional(ps, "scale", 1), out = optional(pout, "out", 2);
    const int64_t M = x.size(0), K = x.size(1), N = w.size(-2), G = offsets.defined() ? w.size(0) : 1;
    if (offsets.defined()) {
      is_dense(w, "w", at::kChar, x, {G, N, K});
      is_dense(ws, "w_scale", at::kFloat, x, {G, N});
      is_dense(offsets, "offsets", at::kInt, x, {G + 1});
    } else {
      is_dense(w, "w", at::kChar, x, {N, K});
      is_dense(ws, "w_scale", at::kFloat, x, {N});
    }
    if (type < 0) type = out.defined() ? dtype_of(out) : scale.defined() ? TOPOEP_BF16 : dtype_of(x);
    if (type < 0) refuse(PyExc_TypeError, "x (or out) must be float32, bfloat16 or float16");
    const at::ScalarType as = type == TOPOEP_F32 ? at::kFloat : type == TOPOEP_BF16 ? at::kBFloat16 : at::kHalf;
    const topoep_int8 p{fits(N), fits(K), fits(G), gated, type};
    size_t need = 0;
    check(entry.int8_bytes(&p, fits(M), &need));
    const bool keep = out.defined(), asked = watched({&x, &scale, &ws});
    if (keep) {
      if (asked || out.requires_grad())
        refuse(PyExc_RuntimeError, "out cannot be given where a gradient is asked for: matmul_int8 is forward only");
      is_dense(out, "out", as, x, {M, gated ? N / 2 : N});
    }
    if (scale.defined()) {
      is_dense(scale, "scale", at::kFloat, x, {M});
      if (x.scalar_type() != at::kChar) refuse(PyExc_TypeError, "q must be int8");
    }
    Tensor q = x;
    if (!scale.defined()) quantize(x, q, scale, st);
    const int64_t ldq = stride_of(q, "q");
    if (!keep) out = at::empty({M, gated ? N / 2 : N}, x.options().dtype(as));
    const Tensor work = scratch(need, x);
    check(entry.int8(&p, q.data_ptr<int8_t>(), ldq, scale.data_ptr<float>(), fits(M),
                     offsets.defined() ? offsets.data_ptr<int32_t>() : nullptr, keep, w.data_ptr<int8_t>(),
                     ws.data_ptr<float>(), out.data_ptr(), work.data_ptr(), (size_t)work.numel(), st));
    if (keep && !out.is_inference()) out.unsafeGetTensorImpl()->bump_version();
    if (asked) out = forward_only(out, "matmul_int8 is forward only: its inputs get no gradient");
    return Py_BuildValue("(iN)", TOPOEP_OK, THPVariable_Wrap(out));
  });
}

PyMethodDef methods[] = {{"bind", bind, METH_VARARGS, "bind(addresses of the library's entries)"},
                         {"expert_rows", expert_rows, METH_VARARGS, "expert_rows(ids, L, slot, stream) -> (code, offsets, pairs, places)"},
                         {"block", block, METH_VARARGS, "block(x, ids, weights, up, down, slot, stream) -> (code, out)"},
                         {"quantize", quantize, METH_VARARGS, "quantize(x, stream) -> (code, q, scale)"},
                         {"matmul_int8", matmul_int8, METH_VARARGS,
                          "matmul_int8(x, scale, w, w_scale, offsets, gated, type, out, stream) -> (code, out)"},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_ffn_tensors", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__ffn_tensors() { return PyModule_Create(&module); }
