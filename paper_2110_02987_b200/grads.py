"""Global norm and clipping of gradients on CUDA tensors the caller owns (no context), in the manner of ``head.py``: calls enqueue on ``stream``
(default: torch's current stream of the tensors' device) and do not wait.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import struct

from . import head
from .binding import GadError
from .head import _ck, _elsewhere, _stream, _switch

_ENTRY = "PiiqqqPq"      # gad_grad_tensor
_ready = False


def _load():
    global _ready
    L = head._load()
    if not _ready:
        L.gad_clip_grads_workspace_bytes.argtypes = [C.c_int64, C.POINTER(C.c_size_t)]
        L.gad_clip_grads.argtypes = [C.c_char_p, C.c_int64, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        _ready = True
    return L


@functools.lru_cache(maxsize=64)
def _packer(n):
    return struct.Struct("@" + _ENTRY * n)


@functools.lru_cache(maxsize=64)
def _workspace(n):
    b = C.c_size_t(0)
    _ck(_load().gad_clip_grads_workspace_bytes(n, C.byref(b)), "gad_clip_grads_workspace_bytes")
    return b.value


def _rows(t, name):
    """(order, rows, cols, row stride) of a dense tensor (order 0), of a matrix with rows (1) or columns (2) that are contiguous."""
    if t.is_contiguous():
        n = t.numel()
        return 0, 1, n, n
    if t.dim() == 2:
        (r, c), (a, b) = t.shape, t.stride()
        if (b == 1 or c == 1) and (a >= c or r == 1):
            return 1, r, c, a
        if (a == 1 or r == 1) and (b >= r or c == 1):
            return 2, c, r, b
    raise GadError(-1, "%s must be contiguous, or a matrix with contiguous rows or columns that do not overlap" % name)


def _entry(t, o, device, types):
    if t.dtype not in types or t.device != device:
        raise GadError(-1, "gradients must be float32, float16 or bfloat16 CUDA tensors on one device")
    order, rows, cols, ld = _rows(t, "a gradient")
    if o is None:
        return t.data_ptr(), types[t.dtype], 0, rows, cols, ld, 0, 0
    if o is t:
        return t.data_ptr(), types[t.dtype], types[t.dtype], rows, cols, ld, t.data_ptr(), ld
    if o.shape != t.shape or o.device != device or (o.dtype is not t.dtype and o.dtype is not head.torch.float32):
        raise GadError(-1, "out must have the gradients' shapes, and their types or float32, on their device")
    oorder, orows, ocols, old = _rows(o, "out")
    if order != oorder:
        if t.dim() == 2 and t.shape[0] == 1:
            # one row, whose values lie apart on one side: columns of one value
            return t.data_ptr(), types[t.dtype], types[o.dtype], t.shape[1], 1, t.stride(1), o.data_ptr(), o.stride(1)
        # a dense matrix has contiguous rows too
        if order + oorder != 1:
            raise GadError(-1, "a gradient and its out must both have contiguous rows, or both contiguous columns")
        rows, cols = t.shape
        ld, old = (ld if order else cols), (old if oorder else cols)
    return t.data_ptr(), types[t.dtype], types[o.dtype], rows, cols, ld, o.data_ptr(), old


def _clip(grads, max_norm, out, stream):
    L = _load()
    if isinstance(grads, head.torch.Tensor) or isinstance(out, head.torch.Tensor):
        raise GadError(-1, "gradients (and out) come as a list of tensors")
    grads = list(grads)
    targets = [None] * len(grads) if out is None else list(out)
    if len(targets) != len(grads):
        raise GadError(-1, "out must have a tensor for every gradient")
    pairs = [(g, o) for g, o in zip(grads, targets) if g is not None]
    if not pairs:
        raise GadError(-1, "there is no gradient")
    dev = pairs[0][0].device
    if dev.type != "cuda":
        raise GadError(-1, "gradients must be float32, float16 or bfloat16 CUDA tensors on one device")
    values, types = [], head._DTYPES
    for g, o in pairs:
        t = types.get(g.dtype)
        if t is not None and (o is g or (o is not None and o.dtype is g.dtype and o.shape == g.shape and o.device == dev and o.is_contiguous())) and g.device == dev and g.is_contiguous():
            n = g.numel()                                        # (most are like this)
            values += (g.data_ptr(), t, t, 1, n, n, o.data_ptr(), n)
        else:
            values += _entry(g, o, dev, types)
    max_norm = float(max_norm)
    if not max_norm >= 0:
        raise GadError(-1, "max_norm must be 0 or more")
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return _launch(L, pairs, values, max_norm, dev)
    return _launch(L, pairs, values, max_norm, dev)


def _launch(L, pairs, values, max_norm, dev):
    n = len(pairs)
    like = pairs[0][0]
    norm = like.new_empty(1, dtype=head.torch.float32)
    nbytes = _workspace(n)
    ws = like.new_empty(nbytes, dtype=head.torch.uint8)
    _ck(L.gad_clip_grads(_packer(n).pack(*values), n, max_norm, norm.data_ptr(), ws.data_ptr(), nbytes, _stream(dev)), "gad_clip_grads")
    return norm


def grad_norm(grads, *, stream=None):
    """gad_clip_grads without clipping: the norm over all values of a list of CUDA tensors (None is passed over), float32 [1]."""
    return _clip(grads, math.inf, None, stream)


def clip_grads(grads, max_norm, *, out=None, stream=None):
    """gad_clip_grads: scales the tensors of a list (None is passed over) by min(1, max_norm / their norm over all values), and returns that norm
    (before clipping), float32 [1].

    float32, float16 or bfloat16 (each its own), contiguous or matrices with a row stride.  In place; with ``out``, a list of tensors of the same shapes, in the
    gradients' types or float32, what is scaled goes there instead.  A norm that is not finite leaves the values as they are.  Autograd does not see the call: the version counters of
    the tensors that it writes stay as they were, so a tensor that a graph has saved must not be among them."""
    grads = list(grads) if not isinstance(grads, head.torch.Tensor if head.torch else ()) else grads
    return _clip(grads, max_norm, grads if out is None else out, stream)
