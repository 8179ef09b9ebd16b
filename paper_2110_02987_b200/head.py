"""Operators of an output head on CUDA tensors the caller owns (no context): layer norm and its backward pass.

Like the rest of the binding this is argument checking and marshalling; the work is the library's kernels (``include/gad.h``).
Every call enqueues on ``stream`` (default: torch's current stream of the tensors' device) and does not wait.  Outputs and
workspaces are allocated per call from torch's allocator on that stream, so calls on different streams, and captured graphs, share nothing.
"""
from __future__ import annotations

import contextlib
import ctypes as C

from .binding import GAD_OK, GadError, load

_DTYPES = {}     # torch dtype -> GAD_F32 / GAD_F16 / GAD_BF16, filled on first use (torch is imported late, as in the rest of the binding)
_lib = None


def _load():
    global _lib
    if _lib is None:
        import torch
        L = load()
        vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float
        L.gad_layer_norm.argtypes = [vp, i64, i64, i32, i32, vp, vp, i32, f32, vp, i64, vp, vp, vp]
        L.gad_layer_norm_backward_workspace_bytes.argtypes = [i64, i32, C.POINTER(C.c_size_t)]
        L.gad_layer_norm_backward.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i32, vp, vp, vp, i64, vp, vp, vp, C.c_size_t, vp]
        _DTYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
        _lib = L
    return _lib


def _matrix(t, name, device=None, shape=None):
    """Checks a row-major CUDA matrix; returns its row stride."""
    if t.dim() != 2 or t.dtype not in _DTYPES or not t.is_cuda:
        raise GadError(-1, "%s must be a float32, float16 or bfloat16 CUDA matrix" % name)
    if device is not None and t.device != device:
        raise GadError(-1, "%s is on another device" % name)
    if shape is not None and tuple(t.shape) != shape:
        raise GadError(-1, "%s must be %d x %d" % ((name,) + shape))
    rows, cols = t.shape
    if cols < 1 or (cols > 1 and t.stride(1) != 1):
        raise GadError(-1, "%s must have at least one column, and its rows contiguous" % name)
    ld = t.stride(0)
    if rows <= 1:
        return max(ld, cols)
    if ld != 0 and ld < cols:
        raise GadError(-1, "the rows of %s overlap" % name)
    return ld


def _vector(t, name, n, dtypes, device):
    """Checks a contiguous CUDA vector of n elements (None passes); returns its address or None."""
    if t is None:
        return None
    if not (t.is_cuda and t.device == device and t.dtype in dtypes and t.dim() == 1 and t.shape[0] == n and (n <= 1 or t.stride(0) == 1)):
        raise GadError(-1, "%s must be a contiguous vector of %d elements (%s) on the same device" % (name, n, " or ".join(str(d) for d in dtypes)))
    return t.data_ptr()


@contextlib.contextmanager
def _switch(device, stream):
    import torch
    with torch.cuda.device(device):
        if stream is None:
            yield torch.cuda.current_stream(device)
        else:
            if stream.device != device:
                raise GadError(-1, "the stream belongs to another device")
            with torch.cuda.stream(stream):     # what is allocated belongs to the stream that uses it
                yield stream


class _Here:
    """The common case: the tensors' device is current and so is the stream."""

    def __init__(self, stream):
        self.stream = stream

    def __enter__(self):
        return self.stream

    def __exit__(self, *a):
        return False


def _on(device, stream):
    import torch
    if stream is None and device.index == torch.cuda.current_device():
        return _Here(torch.cuda.current_stream(device))
    return _switch(device, stream)


def _ck(rc, what):
    if rc != GAD_OK:
        raise GadError(rc, what)


def layer_norm(x, gamma=None, beta=None, *, eps=1e-5, stream=None):
    """gad_layer_norm: ``(y, mean, rstd)`` of the rows of ``x`` [rows x cols]: y = (x - mean) * rstd * gamma + beta.

    x float32, float16 or bfloat16 with any row stride; gamma and beta [cols] in x's type or float32 (both in the same), or None.
    y has x's type and is contiguous; mean and rstd are float32 [rows] (``layer_norm_backward`` takes them)."""
    import torch
    L = _load()
    ldx = _matrix(x, "x")
    rows, cols = x.shape
    params = gamma if gamma is not None else beta
    ptype = x.dtype if params is None else params.dtype
    if ptype is not x.dtype and ptype is not torch.float32:
        raise GadError(-1, "gamma and beta must have x's type or float32")
    g = _vector(gamma, "gamma", cols, (ptype,), x.device)
    b = _vector(beta, "beta", cols, (ptype,), x.device)
    with _on(x.device, stream) as st:
        y = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        stats = torch.empty((2, rows), dtype=torch.float32, device=x.device)
        at = stats.data_ptr()
        _ck(L.gad_layer_norm(x.data_ptr(), ldx, rows, cols, _DTYPES[x.dtype], g, b, _DTYPES[ptype], eps, y.data_ptr(), cols, at, at + 4 * rows,
                             st.cuda_stream), "gad_layer_norm")
    return y, stats[0], stats[1]


def layer_norm_backward(dy, x, mean, rstd, gamma=None, *, param_grads=True, stream=None):
    """gad_layer_norm_backward: ``(dx, dgamma, dbeta)`` for the upstream gradient ``dy`` of ``layer_norm(x, gamma, beta)``.

    dx has x's type, dgamma and dbeta gamma's (x's without one); with ``param_grads=False`` they are None."""
    import torch
    L = _load()
    ldx = _matrix(x, "x")
    rows, cols = x.shape
    lddy = _matrix(dy, "dy", x.device, (rows, cols))
    if dy.dtype is not x.dtype:
        raise GadError(-1, "dy must have x's type")
    ptype = x.dtype if gamma is None else gamma.dtype
    if ptype is not x.dtype and ptype is not torch.float32:
        raise GadError(-1, "gamma must have x's type or float32")
    g = _vector(gamma, "gamma", cols, (ptype,), x.device)
    m = _vector(mean, "mean", rows, (torch.float32,), x.device)
    r = _vector(rstd, "rstd", rows, (torch.float32,), x.device)
    if m is None or r is None:
        raise GadError(-1, "mean and rstd of the forward pass are needed")
    with _on(x.device, stream) as st:
        dx = torch.empty((rows, cols), dtype=x.dtype, device=x.device)
        dgamma = dbeta = ws = None
        nbytes = C.c_size_t(0)
        if param_grads:
            both = torch.empty((2, cols), dtype=ptype, device=x.device)
            dgamma, dbeta = both[0], both[1]
            _ck(L.gad_layer_norm_backward_workspace_bytes(rows, cols, C.byref(nbytes)), "gad_layer_norm_backward_workspace_bytes")
            ws = torch.empty(nbytes.value, dtype=torch.uint8, device=x.device)
        _ck(L.gad_layer_norm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, rows, cols, _DTYPES[x.dtype], g, _DTYPES[ptype], m, r, dx.data_ptr(), cols,
                                      dgamma.data_ptr() if param_grads else None, dbeta.data_ptr() if param_grads else None,
                                      ws.data_ptr() if param_grads else None, nbytes.value, st.cuda_stream), "gad_layer_norm_backward")
    return dx, dgamma, dbeta
