"""Gated feed-forward block on CUDA tensors the caller owns (no context), with its backward pass: the hidden block of a student in front of the
output head (``head.py``), whose manner it shares: calls enqueue on ``stream`` (default: torch's current stream of the tensors' device) and do
not wait, outputs and workspaces are allocated per call, and autograd does not see the calls.
"""
from __future__ import annotations

import ctypes as C
from typing import NamedTuple, Optional

from . import head
from .binding import GadError
from .head import _ck, _elsewhere, _matrix, _stream, _switch

_ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}
_ready = False


class _ForwardArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("cols", C.c_int32), ("inner", C.c_int32), ("activation", C.c_int32), ("rows", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w_gate", C.c_void_p), ("ldwg", C.c_int64), ("w_up", C.c_void_p), ("ldwu", C.c_int64), ("w_down", C.c_void_p), ("ldwd", C.c_int64), ("y", C.c_void_p),
                ("ldy", C.c_int64), ("act", C.c_void_p), ("ldact", C.c_int64), ("slope", C.c_void_p), ("ldslope", C.c_int64), ("h", C.c_void_p), ("ldh", C.c_int64),
                ("status", C.c_void_p)]


class _BackwardArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("cols", C.c_int32), ("inner", C.c_int32), ("rows", C.c_int64), ("dy", C.c_void_p), ("lddy", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64),
                ("w_gate", C.c_void_p), ("ldwg", C.c_int64), ("w_up", C.c_void_p), ("ldwu", C.c_int64), ("w_down", C.c_void_p), ("ldwd", C.c_int64), ("act", C.c_void_p),
                ("ldact", C.c_int64), ("slope", C.c_void_p), ("ldslope", C.c_int64), ("h", C.c_void_p), ("ldh", C.c_int64), ("dx", C.c_void_p), ("lddx", C.c_int64),
                ("dw_gate", C.c_void_p), ("lddwg", C.c_int64), ("dw_up", C.c_void_p), ("lddwu", C.c_int64), ("dw_down", C.c_void_p), ("lddwd", C.c_int64), ("status", C.c_void_p)]


def _load():
    global _ready
    L = head._load()
    if not _ready:
        for name, args in (("gad_gated_feed_forward", _ForwardArgs), ("gad_gated_feed_forward_backward", _BackwardArgs)):
            getattr(L, name + "_workspace_bytes").argtypes = [C.POINTER(args), C.POINTER(C.c_size_t)]
            getattr(L, name).argtypes = [C.POINTER(args), C.c_void_p, C.c_size_t, C.c_void_p]
        _ready = True
    return L


class GatedForward(NamedTuple):
    """What ``gated_feed_forward`` returns.  ``y`` [rows x cols]; ``act``, ``slope`` and ``h`` [rows x inner] for the backward pass, or None;
    ``status`` int32 [1], zero unless a wait inside a kernel ran out."""
    y: "object"
    act: Optional["object"]
    slope: Optional["object"]
    h: Optional["object"]
    status: "object"

    def check(self):
        """Waits for the result; raises GAD_ERR_DEVICE_TIMEOUT if a bounded wait ran out."""
        return _check(self)


class GatedGrads(NamedTuple):
    """What ``gated_feed_forward_backward`` returns: the gradients in the type of x, or None where not asked for, and ``status``."""
    dx: Optional["object"]
    dWg: Optional["object"]
    dWu: Optional["object"]
    dWd: Optional["object"]
    status: "object"

    def check(self):
        """Waits for the result; raises GAD_ERR_DEVICE_TIMEOUT if a bounded wait ran out."""
        return _check(self)


def _check(r):
    code = int(r.status.item())
    if code:
        raise GadError(-7, "wait %d ran out" % code)
    return r


def _weights(x, Wg, Wu, Wd):
    """Checks x and the weights; returns their row strides and the width inside."""
    ldx = _matrix(x, "x")
    cols = x.shape[1]
    ldwg = _matrix(Wg, "Wg", x.device)
    inner = Wg.shape[0]
    if inner < 1 or Wg.shape[1] != cols:
        raise GadError(-1, "Wg must have x's number of columns, and a row at least")
    if inner > head._MOST:
        raise GadError(-2, "Wg has too many rows")
    ldwu = _matrix(Wu, "Wu", x.device, (inner, cols))
    ldwd = _matrix(Wd, "Wd", x.device, (cols, inner))
    if Wg.dtype is not x.dtype or Wu.dtype is not x.dtype or Wd.dtype is not x.dtype:
        raise GadError(-1, "the weights must have x's type")
    if (inner > 1 and (ldwg == 0 or ldwu == 0)) or (cols > 1 and ldwd == 0):
        raise GadError(-1, "the weights must have rows of their own")
    return ldx, ldwg, ldwu, ldwd, inner


_sizes = {}     # what a workspace's size depends on -> its bytes (asking for them is a tenth of a small call)


def _run(ask, call, a, key, like):
    at = C.byref(a)
    nbytes = _sizes.get(key)
    if nbytes is None:
        n = C.c_size_t(0)
        _ck(ask(at, C.byref(n)), call.__name__)
        if len(_sizes) >= 1024:
            _sizes.clear()
        nbytes = _sizes[key] = n.value
    ws = like.new_empty(nbytes, dtype=head.torch.uint8)     # (torch's blocks start on 512 bytes)
    _ck(call(at, ws.data_ptr(), nbytes, _stream(like.device)), call.__name__)


def gated_feed_forward(x, Wg, Wu, Wd, *, activation="silu", save=False, stream=None):
    """gad_gated_feed_forward: ``y = (act(x Wg^T) * (x Wu^T)) Wd^T`` as a ``GatedForward``.

    x [rows x cols], Wg and Wu [inner x cols], Wd [cols x inner], all float32, float16 or bfloat16 (the same), any row stride.  activation: "silu",
    "gelu" (by erf), "relu" or "sigmoid".  With ``save`` the result holds what ``gated_feed_forward_backward`` needs: act(g), u act'(g) and h = act(g) u in x's
    type, in rows that start on 16 bytes.  In float16 an h above 65 504 is infinite."""
    L = _load()
    ldx, ldwg, ldwu, ldwd, inner = _weights(x, Wg, Wu, Wd)
    if activation not in _ACTIVATIONS:
        raise GadError(-1, "activation is one of %s" % ", ".join(_ACTIVATIONS))
    if _elsewhere(x.device, stream):
        with _switch(x.device, stream):
            return gated_feed_forward(x, Wg, Wu, Wd, activation=activation, save=save)
    rows, cols = x.shape
    y = x.new_empty((rows, cols))
    status = x.new_empty(1, dtype=head.torch.int32)
    act = slope = h = None
    at = [None, None, None]
    wide = -(-inner // 8) * 8
    if save:
        act, slope, h = (t[:, :inner] for t in x.new_empty((3, rows, wide)).unbind(0))
        at = [act.data_ptr(), slope.data_ptr(), h.data_ptr()]
    dt, px, pg, pu, pd = head._DTYPES[x.dtype], x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr()
    a = _ForwardArgs(dt, cols, inner, _ACTIVATIONS[activation], rows, px, ldx, pg, ldwg, pu, ldwu, pd, ldwd, y.data_ptr(), cols, at[0], wide, at[1], wide, at[2], wide, status.data_ptr())
    _run(L.gad_gated_feed_forward_workspace_bytes, L.gad_gated_feed_forward, a,
         (dt, rows, cols, inner, save, ldx, ldwg, ldwu, ldwd, px & 15, pg & 15, pu & 15, pd & 15), x)
    return GatedForward(y, act, slope, h, status)


def gated_feed_forward_backward(dy, x, Wg, Wu, Wd, act, slope, h, *, grads=True, stream=None):
    """gad_gated_feed_forward_backward: gradients for the upstream gradient ``dy`` of y, from what ``gated_feed_forward(..., save=True)`` has left, as
    ``GatedGrads``.  grads: True, or some of "x", "g", "u", "d" as a string or set (the gradients of x, Wg, Wu and Wd)."""
    L = _load()
    ldx, ldwg, ldwu, ldwd, inner = _weights(x, Wg, Wu, Wd)
    rows, cols = x.shape
    lddy = _matrix(dy, "dy", x.device, (rows, cols))
    lda, lds, ldh = (_matrix(t, name, x.device, (rows, inner)) for t, name in ((act, "act"), (slope, "slope"), (h, "h")))
    if any(t.dtype is not x.dtype for t in (dy, act, slope, h)):
        raise GadError(-1, "dy, act, slope and h must have x's type")
    if rows > 1 and (lda == 0 or lds == 0 or ldh == 0):
        raise GadError(-1, "act, slope and h must have rows of their own")
    want = {"x", "g", "u", "d"} if grads is True else set() if not grads else set(grads)
    if not want <= {"x", "g", "u", "d"}:
        raise GadError(-1, "grads is True or some of x, g, u and d")
    if _elsewhere(x.device, stream):
        with _switch(x.device, stream):
            return gated_feed_forward_backward(dy, x, Wg, Wu, Wd, act, slope, h, grads=grads)
    dx = x.new_empty((rows, cols)) if "x" in want else None
    dWg = x.new_empty((inner, cols)) if "g" in want else None
    dWu = x.new_empty((inner, cols)) if "u" in want else None
    dWd = x.new_empty((cols, inner)) if "d" in want else None
    status = x.new_empty(1, dtype=head.torch.int32)
    at = [t.data_ptr() if t is not None else None for t in (dx, dWg, dWu, dWd)]
    dt, py, px, pg, pu, pd, ph = head._DTYPES[x.dtype], dy.data_ptr(), x.data_ptr(), Wg.data_ptr(), Wu.data_ptr(), Wd.data_ptr(), h.data_ptr()
    a = _BackwardArgs(dt, cols, inner, rows, py, lddy, px, ldx, pg, ldwg, pu, ldwu, pd, ldwd, act.data_ptr(), lda, slope.data_ptr(), lds, ph, ldh,
                      at[0], cols, at[1], cols, at[2], cols, at[3], inner, status.data_ptr())
    _run(L.gad_gated_feed_forward_backward_workspace_bytes, L.gad_gated_feed_forward_backward, a,
         (dt, rows, cols, inner, None, dx is None, dWg is None, dWu is None, dWd is None, lddy, ldx, ldwg, ldwu, ldwd, ldh, py & 15, px & 15, pg & 15, pu & 15, pd & 15, ph & 15), x)
    return GatedGrads(dx, dWg, dWu, dWd, status)
