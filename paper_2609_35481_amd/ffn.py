"""Thin Python binding of the experts' products (include/topoep_ffn.h).

  feed_forward   the gated feed-forward block (SwiGLU), dense: a shared expert
  experts        the same for the experts a router chose (moe.route's ids and
                 weights), summed by its weights; both are differentiable
  expert_rows    a router's choices in the order of their experts
  quantize       rows in 8-bit integers, a scale each
  matmul_int8    products in 8-bit integers, for all rows or those of every expert

A backward pass is captured into a graph as any other of torch's: with no eager
graph of the same leaves alive, whose accumulators would run on the stream that made them.
What it was given may come through hooks on saved tensors (from the host, computed again), in any
layout; another shape, type or device than was saved is a RuntimeError.

Argument checks and marshalling only: torch provides device memory and the
current stream, every step runs in the HIP kernels of libtopoep.so.  Importing
this module fails loudly when the library, or _ffn_tensors (the calls that take
torch's C++ tensors), has not been built.
"""
from __future__ import annotations

import ctypes

import torch

from .moe import _check, _int32, _on_stream, _stream_of, _TYPES
from .topoep import _lib
from . import _ffn_tensors as _tensors

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


_tensors.bind(*(ctypes.cast(getattr(_lib, _name), _vp).value for _name in EXPORTS))


def _call(name, got):
    """What a call of the library gave; its name is for the error."""
    _check(got[0], name)
    return got[1] if len(got) == 2 else got[1:]


def _queue(*tensors):
    """The stream for tensors' calls; what is no tensor, or on no GPU, the call itself refuses."""
    t = tensors[0]
    return _stream_of(t.device) if isinstance(t, torch.Tensor) and t.is_cuda else 0


def expert_rows(ids, L, expert_slot=None, stream=None):
    """Enqueue topoep_expert_rows for the ids [T, k] of moe.route and the L
    experts that are here: (offsets int32 [L + 1], pairs int32 [T * k], places
    int32 [T, k]).  Slot s has the rows offsets[s] .. offsets[s + 1] - 1;
    pairs names each row's choice t * k + j, places each choice's row, -1 where there is none.
    expert_slot int32 [E] says where an expert lies among the L (-1:
    elsewhere); None: expert e at slot e."""
    if stream is not None:
        return _on_stream(stream, expert_rows, ids, L, expert_slot)
    return _call("topoep_expert_rows", _tensors.expert_rows(ids, _int32("L", L), expert_slot, _queue(ids)))


def feed_forward(x, up, down, stream=None):
    """Enqueue the gated feed-forward block for the rows x [T, H]: down
    (silu(gate x) * (up' x)) with up [2I, H] (I gate rows, then I up rows) and down [H,
    I], bfloat16 or float16.  Differentiable in all three; for the backward
    pass it keeps 10 I bytes a row."""
    if stream is not None:
        return _on_stream(stream, feed_forward, x, up, down)
    return _call("topoep_ffn_forward", _tensors.block(x, None, None, up, down, None, _queue(x)))


def experts(x, ids, weights, up, down, expert_slot=None, stream=None):
    """Enqueue the experts of a routed layer for the tokens x [T, H]: the sum
    over a token's choices (moe.route's ids [T, k] and weights [T, k]) of weight
    times the block of that expert, up [L, 2I, H] and down [L, H, I], bfloat16 or
    float16.  expert_slot int32 [E] says where an expert lies among the L here
    (-1: elsewhere; it adds nothing); None: expert e at slot e.  Differentiable in x,
    weights, up and down; for the backward pass it keeps 10 I bytes for each of T k rows, whether
their experts are here or not."""
    if stream is not None:
        return _on_stream(stream, experts, x, ids, weights, up, down, expert_slot)
    if ids is None:
        raise TypeError("ids is not a tensor")
    return _call("topoep_ffn_forward", _tensors.block(x, ids, weights, up, down, expert_slot, _queue(x)))


def quantize(x, stream=None):
    """Enqueue topoep_quantize: (q int8 [M, K], scale float32 [M]) of the rows x
    [M, K], float32, bfloat16 or float16; x is about q * scale.  A weight matrix's rows are
    its channels.  Forward only."""
    if stream is not None:
        return _on_stream(stream, quantize, x)
    return _call("topoep_quantize", _tensors.quantize(x, _queue(x)))


def matmul_int8(x, w, w_scale, offsets=None, gated=False, dtype=None, out=None, stream=None):
    """Enqueue topoep_matmul_int8: the rows x [M, K] times the weights w int8 [N,
    K] with the scales w_scale float32 [N] of its rows, as quantize makes them.  K is a multiple of 16, at most 2^17.

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
    scale = None
    if isinstance(x, (tuple, list)):
        if len(x) != 2:
            raise ValueError("x is a tensor, or quantize's (q, scale)")
        x, scale = x
        if scale is None:
            raise TypeError("scale is not a tensor")
    if isinstance(gated, torch.Tensor):
        raise TypeError("gated must be true or false, not a tensor")
    if dtype is not None and dtype not in _TYPES:
        raise TypeError("the result must be float32, bfloat16 or float16, not %s" % dtype)
    return _call("topoep_matmul_int8", _tensors.matmul_int8(x, scale, w, w_scale, offsets, bool(gated),
                                                            -1 if dtype is None else _TYPES[dtype], out, _queue(x)))
