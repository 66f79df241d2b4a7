"""Thin Python binding of the experts' products (include/topoep_ffn.h).

  feed_forward   the gated feed-forward block (SwiGLU), dense: a shared expert
  experts        the same for the experts a router chose (moe.route's ids and
                 weights), summed by its weights; both are differentiable
  expert_rows    a router's choices in the order of their experts
  quantize       rows in 8-bit integers, a scale each
  matmul_int8    products in 8-bit integers, for all rows or those of every expert

Argument checks and marshalling only: torch provides device memory and the
current stream, every step runs in the HIP kernels of libtopoep.so.  Importing
this module fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes
import functools

import torch

from .moe import _check, _dense, _int32, _on_stream, _stream_of, _TYPES
from .topoep import _lib

MAX_EXPERTS = 1024


class Ffn(ctypes.Structure):
    """topoep_ffn: H, I, the blocks of weights and their type."""
    _fields_ = [("hidden", ctypes.c_int32), ("inter", ctypes.c_int32), ("experts", ctypes.c_int32),
                ("dtype", ctypes.c_int32)]


class Rows(ctypes.Structure):
    """topoep_ffn_rows: where the rows of the experts are, and k."""
    _fields_ = [("offsets", ctypes.c_void_p), ("pairs", ctypes.c_void_p), ("places", ctypes.c_void_p),
                ("weights", ctypes.c_void_p), ("topk", ctypes.c_int32), ("num_experts", ctypes.c_int32)]


class Int8(ctypes.Structure):
    """topoep_int8: N, K, the weight matrices, whether they are gated, the output's type."""
    _fields_ = [("n", ctypes.c_int32), ("k", ctypes.c_int32), ("groups", ctypes.c_int32), ("gated", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32)]


_vp, _i32, _i64, _size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
_PF, _PR, _P8, _PS = (ctypes.POINTER(t) for t in (Ffn, Rows, Int8, _size))
for _name, _args in (
        ("topoep_expert_rows_workspace_bytes", [_i32, _i32, _i32, _PS]),
        ("topoep_expert_rows", [_vp, _i32, _i32, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _size, _vp]),
        ("topoep_ffn_bytes", [_PF, _i32, _PR, _PS, _PS, _PS]),
        ("topoep_ffn_forward", [_PF, _vp, _i64, _i32, _PR, _vp, _vp, _vp, _vp, _vp, _size, _vp]),
        ("topoep_ffn_backward", [_PF, _vp, _i64, _i32, _PR, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _size, _vp]),
        ("topoep_quantize", [_vp, _i32, _i64, _i32, _i32, _vp, _vp, _vp]),
        ("topoep_matmul_int8_workspace_bytes", [_P8, _i32, _PS]),
        ("topoep_matmul_int8", [_P8, _vp, _i64, _vp, _i32, _vp, _i32, _vp, _vp, _vp, _vp, _size, _vp])):
    _fn = getattr(_lib, _name)
    _fn.restype, _fn.argtypes = ctypes.c_int, _args

EXPORTS = ("topoep_expert_rows_workspace_bytes", "topoep_expert_rows", "topoep_ffn_bytes", "topoep_ffn_forward",
           "topoep_ffn_backward", "topoep_quantize", "topoep_matmul_int8_workspace_bytes", "topoep_matmul_int8")


def _tensor(t, name, dims):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s is not a tensor" % name)
    if t.dim() != dims:
        raise ValueError("%s must have %d dimensions, got %s" % (name, dims, tuple(t.shape)))
    if torch.autograd.forward_ad._current_level >= 0 and torch.autograd.forward_ad.unpack_dual(t).tangent is not None:
        raise RuntimeError("%s carries a tangent, which is not passed on" % name)
    return t


def _row_stride(t, name):
    """Of a matrix of dense rows that do not overlap."""
    rows, cols = t.shape
    if (cols > 1 and t.stride(1) != 1) or (rows > 1 and t.stride(0) < cols):
        raise ValueError("%s must be a matrix of dense rows that do not overlap" % name)
    return t.stride(0) if rows > 1 else (cols + 15) // 16 * 16


def _watched(*tensors):
    return torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad for t in tensors)


def _bytes(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device)   # torch aligns to 512 bytes


def _at(t):
    return None if t is None else t.data_ptr()


# ---------------------------------------------------------------- rows by expert

@functools.lru_cache(maxsize=256)
def _rows_workspace(T, k, L):
    out = _size(0)
    _check(_lib.topoep_expert_rows_workspace_bytes(T, k, L, out), "topoep_expert_rows_workspace_bytes")
    return out.value


def expert_rows(ids, L, expert_slot=None, stream=None):
    """Enqueue topoep_expert_rows for the ids [T, k] of moe.route and the L
    experts that are here: (offsets int32 [L + 1], pairs int32 [T * k], places
    int32 [T, k]).  Slot s has the rows offsets[s] .. offsets[s + 1] - 1;
    pairs names each row's choice t * k + j, places each choice's row, -1 where there is none.
    expert_slot int32 [E] says where an expert lies among the L (-1:
    elsewhere); None: expert e at slot e."""
    if stream is not None:
        return _on_stream(stream, expert_rows, ids, L, expert_slot)
    L = _int32("L", L)
    queue = _stream_of(_tensor(ids, "ids", 2).device)
    T, k = _int32("T", ids.shape[0]), _int32("k", ids.shape[1])
    dev = _dense(ids, "ids", (T, k), torch.int32, ids.device).device
    E = L
    if expert_slot is not None:
        E = _int32("E", _tensor(expert_slot, "expert_slot", 1).shape[0])
        _dense(expert_slot, "expert_slot", (E,), torch.int32, dev)
    need = _rows_workspace(T, k, L)
    offsets = torch.empty(L + 1, dtype=torch.int32, device=dev)
    pairs, places = torch.empty(T * k, dtype=torch.int32, device=dev), torch.empty_like(ids)
    ws = _bytes(max(need, 1), dev)
    _check(_lib.topoep_expert_rows(ids.data_ptr(), T, k, _at(expert_slot), E, L, offsets.data_ptr(), pairs.data_ptr(),
                                   places.data_ptr(), ws.data_ptr(), ws.numel(), queue), "topoep_expert_rows")
    return offsets, pairs, places


# ---------------------------------------------------------------- the gated block

class _Block:
    """A call's sizes and operands, as the library takes them."""
    def __init__(self, x, up, down, rows, weights, E):
        self.x, self.up, self.down, self.rows, self.weights = x, up, down, rows, weights
        lead = () if rows is None else (up.shape[0],)
        H, I = down.shape[-2], down.shape[-1]
        if x.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("x must be bfloat16 or float16, not %s" % x.dtype)
        if x.shape[1] != H:
            raise ValueError("x is [T, H], up [.., 2I, H], down [.., H, I]: got %s, %s and %s" %
                             (tuple(x.shape), tuple(up.shape), tuple(down.shape)))
        _dense(up, "up", lead + (2 * I, H), x.dtype, x.device)
        _dense(down, "down", lead + (H, I), x.dtype, x.device)
        self.T, self.ldx = _int32("T", x.shape[0]), _row_stride(x, "x")
        self.ffn = Ffn(_int32("H", H), _int32("I", I), _int32("L", lead[0] if lead else 1), _TYPES[x.dtype])
        self.arg = None
        if rows is not None:
            k = _int32("k", rows[2].shape[1])
            _dense(weights, "weights", (self.T, k), torch.float32, x.device)
            self.arg = Rows(*(t.data_ptr() for t in rows), weights.data_ptr(), k, E)
        need = _size(0), _size(0), _size(0)
        _check(_lib.topoep_ffn_bytes(self.ffn, self.T, self.arg, *need), "topoep_ffn_bytes")
        self.forward_bytes, self.saved_bytes, self.backward_bytes = (n.value for n in need)

    def forward(self, keep):
        """(out, what a backward pass needs, or None)"""
        x, queue = self.x, _stream_of(self.x.device)
        out = torch.empty((self.T, self.ffn.hidden), dtype=x.dtype, device=x.device)
        saved = _bytes(self.saved_bytes, x.device) if keep else None
        ws = _bytes(max(self.forward_bytes, 1), x.device)
        _check(_lib.topoep_ffn_forward(self.ffn, x.data_ptr(), self.ldx, self.T, self.arg, self.up.data_ptr(),
                                       self.down.data_ptr(), out.data_ptr(), _at(saved), ws.data_ptr(), ws.numel(),
                                       queue), "topoep_ffn_forward")
        return out, saved

    def backward(self, saved, grad, wants):
        """The gradients of x, weights, up and down that are wanted."""
        x, queue = self.x, _stream_of(self.x.device)
        like = ((x.shape, x.dtype), ((0,) if self.weights is None else self.weights.shape, torch.float32),
                (self.up.shape, x.dtype), (self.down.shape, x.dtype))
        got = [torch.empty(shape, dtype=dtype, device=x.device) if want else None
               for want, (shape, dtype) in zip(wants, like)]
        ws = _bytes(max(self.backward_bytes, 1), x.device)
        _check(_lib.topoep_ffn_backward(self.ffn, x.data_ptr(), self.ldx, self.T, self.arg, self.up.data_ptr(),
                                        self.down.data_ptr(), saved.data_ptr(), grad.data_ptr(), *map(_at, got),
                                        ws.data_ptr(), ws.numel(), queue), "topoep_ffn_backward")
        return got


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weights, up, down, rows, E):
        out, saved = _Block(x, up, down, rows, weights, E).forward(True)
        ctx.num_experts = E
        ctx.save_for_backward(x, weights, up, down, saved, *(rows or ()))
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad):
        x, weights, up, down, saved, *rows = ctx.saved_tensors
        block = _Block(x, up, down, tuple(rows) or None, weights, ctx.num_experts)
        grad = grad.contiguous()
        if grad.data_ptr() % 16:
            grad = grad.clone()
        return (*block.backward(saved, grad, ctx.needs_input_grad[:4]), None, None)


def _run(x, weights, up, down, rows, E):
    if _watched(x, weights, up, down):
        return _FeedForward.apply(x, weights, up, down, rows, E)
    return _Block(x, up, down, rows, weights, E).forward(False)[0]


def feed_forward(x, up, down, stream=None):
    """Enqueue the gated feed-forward block for the rows x [T, H]: down
    (silu(gate x) * (up' x)) with up [2I, H] (I gate rows, then I up rows) and down [H,
    I], bfloat16 or float16.  Differentiable in all three; for the backward
    pass it keeps 10 I bytes a row."""
    if stream is not None:
        return _on_stream(stream, feed_forward, x, up, down)
    _stream_of(_tensor(x, "x", 2).device)
    return _run(x, None, _tensor(up, "up", 2), _tensor(down, "down", 2), None, 1)


def experts(x, ids, weights, up, down, expert_slot=None, stream=None):
    """Enqueue the experts of a routed layer for the tokens x [T, H]: the sum
    over a token's choices (moe.route's ids [T, k] and weights [T, k]) of weight
    times the block of that expert, up [L, 2I, H] and down [L, H, I], bfloat16 or
    float16.  expert_slot int32 [E] says where an expert lies among the L here
    (-1: elsewhere; it adds nothing); None: expert e at slot e.  Differentiable in x,
    weights, up and down; for the backward pass it keeps 10 I bytes for each of T k rows."""
    if stream is not None:
        return _on_stream(stream, experts, x, ids, weights, up, down, expert_slot)
    _stream_of(_tensor(x, "x", 2).device)
    _tensor(up, "up", 3), _tensor(down, "down", 3), _tensor(weights, "weights", 2)
    if _tensor(ids, "ids", 2).shape[0] != x.shape[0] or ids.device != x.device:
        raise ValueError("ids must have a row for each of x, on its GPU")
    rows = expert_rows(ids, up.shape[0], expert_slot)
    E = up.shape[0] if expert_slot is None else expert_slot.shape[0]
    return _run(x, weights, up, down, rows, max(E, 1))


# ---------------------------------------------------------------- 8-bit integers

class _Forward(torch.autograd.Function):
    """A call under autograd that has no gradient: a backward pass through it is
    an error, not nothing."""
    @staticmethod
    def forward(ctx, name, call, *inputs):
        ctx.name = name
        out = call()
        if isinstance(out, tuple):
            ctx.mark_non_differentiable(out[0])
        return out

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("%s is forward only: its inputs get no gradient" % ctx.name)


def quantize(x, stream=None):
    """Enqueue topoep_quantize: (q int8 [M, K], scale float32 [M]) of the rows x
    [M, K], float32, bfloat16 or float16; x is about q * scale.  A weight matrix's rows are
    its channels.  Forward only."""
    if stream is not None:
        return _on_stream(stream, quantize, x)
    if _watched(_tensor(x, "x", 2)):
        return _Forward.apply("quantize", lambda: _quantize(x), x)
    return _quantize(x)


def _quantize(x):
    queue = _stream_of(x.device)
    if x.dtype not in _TYPES:
        raise TypeError("x must be float32, bfloat16 or float16, not %s" % x.dtype)
    M, K = _int32("M", x.shape[0]), _int32("K", x.shape[1])
    q = torch.empty((M, K), dtype=torch.int8, device=x.device)
    scale = torch.empty(M, dtype=torch.float32, device=x.device)
    _check(_lib.topoep_quantize(x.data_ptr(), _TYPES[x.dtype], _row_stride(x, "x"), M, K, q.data_ptr(),
                                scale.data_ptr(), queue), "topoep_quantize")
    return q, scale


def matmul_int8(x, w, w_scale, offsets=None, gated=False, dtype=None, out=None, stream=None):
    """Enqueue topoep_matmul_int8: the rows x [M, K] times the weights w int8 [N,
    K] with the scales w_scale float32 [N] of its rows, as quantize makes them.

    x        float32, bfloat16 or float16, which is quantised row by row first, or what
             quantize returned for it: (q, scale)
    offsets  int32 [G + 1]: matrix g of w [G, N, K] and w_scale [G, N] takes the
             rows offsets[g] .. offsets[g + 1] - 1 (expert_rows makes them)
    gated    w is N / 2 gate rows, then N / 2 up rows: silu(gate) * up
    dtype    of the result [M, N] (gated [M, N / 2]): float32, bfloat16 or float16; None: x's
             (bfloat16 for a pair)
    out      a tensor for the result, whose rows behind the last offset stay as they were;
             None makes one, where they are zeros

    Forward only."""
    if stream is not None:
        return _on_stream(stream, matmul_int8, x, w, w_scale, offsets, gated, dtype, out)
    pair = x if isinstance(x, (tuple, list)) else None
    if pair is not None and len(pair) != 2:
        raise ValueError("x is a tensor, or quantize's (q, scale)")
    if _watched(w_scale, *(pair or (x,))):
        if out is not None:
            raise RuntimeError("out cannot be given where a gradient is asked for: matmul_int8 is forward only")
        return _Forward.apply("matmul_int8", lambda: _matmul_int8(x, w, w_scale, offsets, gated, dtype, None), w_scale,
                              *(pair or (x,)))
    return _matmul_int8(x, w, w_scale, offsets, gated, dtype, out)


def _matmul_int8(x, w, w_scale, offsets, gated, dtype, out):
    pair = x if isinstance(x, (tuple, list)) else None
    _tensor(w, "w", 2 if offsets is None else 3)
    q = _tensor(pair[0] if pair else x, "x", 2)
    dev, queue = q.device, _stream_of(q.device)
    if dtype is None:
        dtype = (torch.bfloat16 if pair else x.dtype) if out is None else out.dtype
    if dtype not in _TYPES:
        raise TypeError("the result must be float32, bfloat16 or float16, not %s" % dtype)
    M, K, N = _int32("M", q.shape[0]), _int32("K", q.shape[1]), _int32("N", w.shape[-2])
    G = 1 if offsets is None else _int32("G", w.shape[0])
    _dense(w, "w", (() if offsets is None else (G,)) + (N, K), torch.int8, dev)
    _dense(w_scale, "w_scale", tuple(w.shape[:-1]), torch.float32, dev)
    if offsets is not None:
        _dense(offsets, "offsets", (G + 1,), torch.int32, dev)
    p = Int8(N, K, G, int(bool(gated)), _TYPES[dtype])
    need = _size(0)
    _check(_lib.topoep_matmul_int8_workspace_bytes(p, M, need), "topoep_matmul_int8_workspace_bytes")
    shape = (M, N // 2 if gated else N)
    keep = out is not None
    if keep:
        if out.requires_grad:
            raise RuntimeError("out asks for a gradient, which matmul_int8 does not have")
        _dense(_tensor(out, "out", 2), "out", shape, dtype, dev)
    if pair:
        scale = _dense(_tensor(pair[1], "scale", 1), "scale", (M,), torch.float32, dev)
        if q.dtype != torch.int8:
            raise TypeError("q must be int8, not %s" % q.dtype)
        ldq = _row_stride(q, "q")
    else:
        q, scale = _quantize(x)
        ldq = K
    if not keep:
        out = torch.empty(shape, dtype=dtype, device=dev)
    ws = _bytes(max(need.value, 1), dev)
    _check(_lib.topoep_matmul_int8(p, q.data_ptr(), ldq, scale.data_ptr(), M, _at(offsets), int(keep), w.data_ptr(),
                                   w_scale.data_ptr(), out.data_ptr(), ws.data_ptr(), ws.numel(), queue),
           "topoep_matmul_int8")
    if keep:
        torch.autograd.graph.increment_version(out)
    return out
