"""Thin Python binding of the operators beside the planner (include/topoep_moe.h).

  route, route_backward   the router: top-k ids (what a planner takes) and
                          weights of every token, and its gradient; route is
                          differentiable where the logits ask for a gradient
  moe_few                 a whole mixture-of-experts layer for up to 128 tokens
  grad_norm, clip_grads   the global gradient norm over many tensors and the
                          clip

Argument checks and marshalling only: torch provides device memory and the
current stream, every step runs in the HIP kernels of libtopoep.so.  Importing this module fails
loudly when the library, or _tensors (the calls that take torch's C++ tensors), has not been built.
"""
from __future__ import annotations

import ctypes
import functools
import numbers

import torch

from .topoep import OK, TopoepError, _lib
from . import _tensors

F32, BF16, F16 = 0, 1, 2
SOFTMAX, SIGMOID = 0, 1
MAX_EXPERTS = 1024
MAX_TOPK = 64
MAX_TOKENS = 128

_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_SCORES = {"softmax": SOFTMAX, "sigmoid": SIGMOID}
_ORDERS = {"2": 0, 2: 0, 2.0: 0, "inf": 1, float("inf"): 1}


class Router(ctypes.Structure):
    """topoep_router: E, k, expert groups, scores and the logits' type."""
    _fields_ = [("num_experts", ctypes.c_int32), ("topk", ctypes.c_int32), ("groups", ctypes.c_int32),
                ("top_groups", ctypes.c_int32), ("scoring", ctypes.c_int32), ("renorm", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


class Moe(ctypes.Structure):
    """topoep_moe: H, I, the experts whose weights are here, their type."""
    _fields_ = [("hidden", ctypes.c_int32), ("inter", ctypes.c_int32), ("local_experts", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class Grad(ctypes.Structure):
    """topoep_grad: one tensor of a gradient set."""
    _fields_ = [("grad", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("out_dtype", ctypes.c_int32)]


_vp, _i32, _i64, _f32, _size = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t)
_PR, _PM, _PS = ctypes.POINTER(Router), ctypes.POINTER(Moe), ctypes.POINTER(_size)
for _name, _args in (
        ("topoep_route", [_PR, _vp, _i64, _i32, _vp, _vp, _vp, _vp]),
        ("topoep_route_backward", [_PR, _vp, _i64, _i32, _vp, _vp, _vp, _i64, _vp]),
        ("topoep_moe_workspace_bytes", [_PM, _PR, _i32, _PS]),
        ("topoep_moe_few", [_PM, _PR, _vp, _i64, _i32, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _size, _vp]),
        ("topoep_grads_workspace_bytes", [_i32, _PS]),
        ("topoep_grad_norm", [_vp, _i32, _f32, _i32, _vp, _vp, _size, _vp]),
        ("topoep_clip_grads", [_vp, _i32, _f32, _i32, _f32, _vp, _vp, _vp, _size, _vp])):
    _fn = getattr(_lib, _name)
    _fn.restype, _fn.argtypes = ctypes.c_int, _args

_ROUTE = ctypes.cast(_lib.topoep_route, _vp).value
_MOE_FEW = ctypes.cast(_lib.topoep_moe_few, _vp).value
_ROUTE_BACKWARD = ctypes.cast(_lib.topoep_route_backward, _vp).value

EXPORTS = ("topoep_route", "topoep_route_backward", "topoep_moe_workspace_bytes", "topoep_moe_few",
           "topoep_grads_workspace_bytes", "topoep_grad_norm", "topoep_clip_grads")


def _int32(name, value):
    """A size as the library's 32 bits take it, which ctypes would cut it to."""
    if not isinstance(value, numbers.Integral):
        raise TypeError("%s must be an integer, not %s" % (name, type(value).__name__))
    if not -2 ** 31 <= value < 2 ** 31:
        raise ValueError("%s is %d, beyond 32 bits" % (name, value))
    return int(value)


@functools.lru_cache(maxsize=256)
def router(E, k, dtype=torch.float32, scoring="softmax", renorm=True, scale=1.0, groups=1, top_groups=1) -> Router:
    """The sizes and rules of a router.  Plain values alone, so that one struct
    serves every call that names the same: a tensor, whose value may change, is
    refused."""
    if not isinstance(scale, numbers.Real):
        raise TypeError("scale must be a number, not %s" % type(scale).__name__)
    if isinstance(renorm, torch.Tensor):
        raise TypeError("renorm must be true or false, not a tensor")
    if dtype not in _TYPES:
        raise TypeError("logits must be float32, bfloat16 or float16, not %s" % dtype)
    if scoring not in _SCORES:
        raise ValueError("scoring is 'softmax' or 'sigmoid', not %r" % (scoring,))
    return Router(_int32("E", E), _int32("k", k), _int32("groups", groups), _int32("top_groups", top_groups),
                  _SCORES[scoring], int(bool(renorm)), _TYPES[dtype], float(scale))


def _check(rc, name):
    if rc != OK:
        raise TopoepError(name, rc)


def _dense(t, name, shape, dtype, device):
    if t.dtype != dtype or t.device != device:
        raise TypeError("%s must be %s on %s" % (name, dtype, device))
    if tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be contiguous of shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t


def _stream_of(device):
    """The current stream of the tensors' device, which has to be the current
    device: the library's calls go there."""
    if device.type != "cuda":
        raise TypeError("tensors must be on a GPU, not on %s" % device)
    if torch._C._cuda_getDevice() != device.index:
        raise ValueError("the tensors are on %s, the current device is cuda:%d" % (device, torch.cuda.current_device()))
    return torch._C._cuda_getCurrentRawStream(device.index)


def _on_stream(stream, call, *args):
    """call(*args) with a stream named by the caller as the current one: what a
    call allocates belongs to the stream its kernels run on."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)))
    with torch.cuda.stream(stream):
        return call(*args)


def _route(r, logits, bias):
    rc, ids, weights = _tensors.route(_ROUTE, ctypes.addressof(r), logits, bias, _stream_of(logits.device))
    _check(rc, "topoep_route")
    return ids, weights


def _backward(r, logits, ids, grad_weights):
    rc, out = _tensors.route_backward(_ROUTE_BACKWARD, ctypes.addressof(r), logits, ids, grad_weights,
                                      _stream_of(logits.device))
    _check(rc, "topoep_route_backward")
    return out


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, bias, r):
        ids, weights = _route(r, logits, bias)
        ctx.save_for_backward(logits, ids)
        ctx.mark_non_differentiable(ids)
        ctx.router = r
        return ids, weights

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, grad_weights):
        logits, ids = ctx.saved_tensors
        return _backward(ctx.router, logits, ids, grad_weights.contiguous()), None, None


class _RouteBackward(torch.autograd.Function):
    """A direct call's result under autograd: a gradient through it is an
    error, not nothing."""
    @staticmethod
    def forward(ctx, logits, ids, grad_weights, r):
        return _backward(r, logits, ids, grad_weights)

    @staticmethod
    def backward(ctx, _):
        raise RuntimeError("route_backward has no gradient of its own")


class _Few(torch.autograd.Function):
    """The layer under autograd: a backward pass through it is an error, not
    one that leaves its weights out."""
    @staticmethod
    def forward(ctx, x, gate, up, down, bias, k, rules, expert_slot, workspace):
        out, ids, weights = _few(x, gate, up, down, k, rules, bias, expert_slot, workspace)
        ctx.mark_non_differentiable(ids)
        return out, ids, weights

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("moe_few is forward only: its inputs get no gradient")


def _watched(*tensors):
    """Whether autograd would record an operation on them."""
    return torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors)


def route(logits, k, scoring="softmax", renorm=True, scale=1.0, bias=None, groups=1, top_groups=1, stream=None):
    """Enqueue topoep_route: (ids int32 [T, k], weights float32 [T, k]) of the
    logits [T, E].  The ids are what a planner takes; the weights carry a
    gradient to logits that require one (a bias gets none).  A bias is added to
    the logits where experts are chosen (a bias trained on sigmoid scores is
    another rule), and a group counts by its largest such sum."""
    r = router(logits.shape[1] if logits.dim() == 2 else 0, k, logits.dtype, scoring, renorm, scale, groups,
               top_groups)
    if stream is not None:
        return _on_stream(stream, route, logits, k, scoring, renorm, scale, bias, groups, top_groups)
    if logits.requires_grad and torch.is_grad_enabled():
        return _Route.apply(logits, bias, r)
    return _route(r, logits, bias)


def route_backward(logits, ids, grad_weights, scoring="softmax", renorm=True, scale=1.0, stream=None):
    """Enqueue topoep_route_backward: the logits' gradient [T, E] in their
    type from the weights' [T, k]."""
    r = router(logits.shape[1] if logits.dim() == 2 else 0, ids.shape[1] if ids.dim() == 2 else 0, logits.dtype,
               scoring, renorm, scale)
    if stream is not None:
        return _on_stream(stream, route_backward, logits, ids, grad_weights, scoring, renorm, scale)
    if _watched(logits, grad_weights):
        return _RouteBackward.apply(logits, ids, grad_weights, r)
    return _backward(r, logits, ids, grad_weights)


def moe_workspace_bytes(H, I, E, L, k, T, dtype=torch.bfloat16) -> int:
    """Bytes of workspace moe_few needs for T tokens or fewer (and up to 255
    more where it does not start at a multiple of 256)."""
    out = _size(0)
    m = Moe(_int32("H", H), _int32("I", I), _int32("L", L), _TYPES.get(dtype, -1))
    _check(_lib.topoep_moe_workspace_bytes(m, router(E, k), _int32("T", T), out), "topoep_moe_workspace_bytes")
    return out.value


def moe_few(x, gate, up, down, k, scoring="softmax", renorm=True, scale=1.0, bias=None, groups=1, top_groups=1,
            expert_slot=None, workspace=None, stream=None):
    """Enqueue topoep_moe_few: (out [T, H], ids int32 [T, k], weights float32
    [T, k]) of the tokens x [T, H], at most 128, through a layer with the
    router gate [E, H] and the experts up [L, 2I, H] (gate rows, then up rows)
    and down [L, H, I], bfloat16 or float16.  expert_slot [E] says where an
    expert lies among the L here (-1: elsewhere; it adds nothing).  Forward
    only: a backward pass through the outputs is an error.

    workspace: a tensor of moe_workspace_bytes or more for calls on one stream to
    share; None makes one for the call."""
    rules = (scoring, renorm, scale, groups, top_groups)
    if stream is not None:
        return _on_stream(stream, moe_few, x, gate, up, down, k, *rules[:3], bias, *rules[3:], expert_slot, workspace)
    if _watched(x, gate, up, down, bias):
        return _Few.apply(x, gate, up, down, bias, k, rules, expert_slot, workspace)
    return _few(x, gate, up, down, k, rules, bias, expert_slot, workspace)


def _few(x, gate, up, down, k, rules, bias, expert_slot, workspace):
    stream = _stream_of(x.device)
    if gate.dim() != 2 or down.dim() != 3 or x.dim() != 2:
        raise ValueError("x is [T, H], gate [E, H], up [L, 2I, H], down [L, H, I]")
    r = router(gate.shape[0], k, torch.float32, *rules)
    if x.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("x must be bfloat16 or float16, not %s" % x.dtype)
    if workspace is None:
        (L, H, I), dtype = down.shape, x.dtype
        workspace = torch.empty(moe_workspace_bytes(H, I, gate.shape[0], L, k, x.shape[0], dtype) + 255,
                                dtype=torch.uint8, device=x.device)
    rc, out, ids, weights = _tensors.moe_few(_MOE_FEW, ctypes.addressof(r), x, gate, up, down, bias, expert_slot,
                                             workspace, stream)
    _check(rc, "topoep_moe_few")
    return out, ids, weights


def _grad_set(grads, outs):
    """The set as the library takes it (topoep_grad after topoep_grad), its
    length and device."""
    table, device = _tensors.pack(grads, outs)
    return table, len(grads), torch.device("cuda", device if device >= 0 else torch.cuda.current_device())


def _order(ord):
    if ord not in _ORDERS:
        raise ValueError("ord is 2 or inf, not %r" % (ord,))
    return _ORDERS[ord]


@functools.lru_cache(maxsize=64)
def grads_workspace_bytes(count) -> int:
    out = _size(0)
    _check(_lib.topoep_grads_workspace_bytes(count, out), "topoep_grads_workspace_bytes")
    return out.value


def grad_norm(grads, scale=1.0, ord=2, stream=None):
    """Enqueue topoep_grad_norm: scale times the 2-norm (or, with ord inf, the
    largest magnitude) over a list of tensors, as a float32 scalar tensor."""
    if stream is not None:
        return _on_stream(stream, grad_norm, grads, scale, ord)
    table, n, dev = _grad_set(grads, None)
    queue = _stream_of(dev)
    norm = torch.empty((), dtype=torch.float32, device=dev)
    ws = torch.empty(grads_workspace_bytes(n), dtype=torch.uint8, device=dev)   # torch aligns to 512 bytes
    _check(_lib.topoep_grad_norm(table, n, scale, _order(ord), norm.data_ptr(), ws.data_ptr(),
                                 ws.numel(), queue), "topoep_grad_norm")
    return norm


def clip_grads(grads, max_norm, scale=1.0, ord=2, outs=None, norm=None, stream=None):
    """Enqueue topoep_clip_grads: every gradient times scale * min(1, max_norm /
    (norm + 1e-6)), in place or into `outs` (same shapes and strides, any
    of the three types), none of which overlaps another tensor of the set but
    its own gradient; returns the norm.  norm: a given one (float32 scalar tensor,
    already scaled), say of a whole group of ranks; None takes this set's.  A norm that
    is not finite leaves every tensor as it is."""
    if stream is not None:
        return _on_stream(stream, clip_grads, grads, max_norm, scale, ord, outs, norm)
    table, n, dev = _grad_set(grads, outs)
    queue = _stream_of(dev)
    total = torch.empty((), dtype=torch.float32, device=dev) if norm is None else \
        _dense(norm, "norm", (), torch.float32, dev)
    ws = torch.empty(grads_workspace_bytes(n), dtype=torch.uint8, device=dev)
    _check(_lib.topoep_clip_grads(table, n, scale, _order(ord), max_norm,
                                  total.data_ptr() if norm is not None else None,
                                  total.data_ptr() if norm is None else None, ws.data_ptr(), ws.numel(), queue),
           "topoep_clip_grads")
    _tensors.written(grads if outs is None else outs)
    return total
