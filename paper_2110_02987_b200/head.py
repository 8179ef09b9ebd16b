"""Operators of an output head on CUDA tensors the caller owns (no context): layer norm and its backward pass, the softmax cross entropy
of an output layer with many classes, distillation from a teacher's top logits, and the clipped policy loss of actions among the classes.

Like the rest of the binding this is argument checking and marshalling; the work is the library's kernels (``include/gad.h``).
Every call enqueues on ``stream`` (default: torch's current stream of the tensors' device) and does not wait.  Outputs and
workspaces are allocated per call from torch's allocator on that stream, so calls on different streams, and captured graphs, share nothing.  As everywhere
in torch, tensors made on another stream must be ready when the call's stream gets there.  The calls record nothing for autograd, whether their inputs require
gradients or not: gradients are what they return, to be handed on (``h.backward(r.dH)`` for an ``h`` that autograd knows).
"""
from __future__ import annotations

import contextlib
import ctypes as C
import functools
from typing import NamedTuple, Optional

from .binding import GAD_OK, GadError, load

_DTYPES = {}     # torch dtype -> GAD_F32 / GAD_F16 / GAD_BF16, filled on first use (torch is imported late, as in the rest of the binding)
_lib = torch = None
_MOST = 2 ** 31 - 1     # the library's columns, classes and slots are 32-bit integers, to which ctypes would cut a longer one without a word


class _ClassLossArgs(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("cols", C.c_int32), ("classes", C.c_int32), ("rows", C.c_int64), ("H", C.c_void_p), ("ldh", C.c_int64),
                ("W", C.c_void_p), ("ldw", C.c_int64), ("bias", C.c_void_p), ("labels", C.c_void_p), ("label_bytes", C.c_int32), ("k", C.c_int32),
                ("target_classes", C.c_void_p), ("target_bytes", C.c_int32), ("teacher_dtype", C.c_int32), ("teacher", C.c_void_p),
                ("temperature", C.c_float), ("hard_weight", C.c_float), ("row_weights", C.c_void_p), ("scale", C.c_float), ("mean", C.c_int32),
                ("loss", C.c_void_p), ("row_loss", C.c_void_p), ("dH", C.c_void_p), ("lddh", C.c_int64), ("dW", C.c_void_p), ("lddw", C.c_int64),
                ("db", C.c_void_p), ("status", C.c_void_p)]


class _PolicyLossArgs(C.Structure):
    _fields_ = [("head", _ClassLossArgs), ("old_logp", C.c_void_p), ("advantages", C.c_void_p), ("ref_logp", C.c_void_p), ("clip_low", C.c_float), ("clip_high", C.c_float),
                ("kl_weight", C.c_float), ("logp", C.c_void_p)]


def _load():
    global _lib, torch
    if _lib is None:
        import torch
        L = load()
        vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float
        L.gad_layer_norm.argtypes = [vp, i64, i64, i32, i32, vp, vp, i32, f32, vp, i64, vp, vp, vp]
        L.gad_layer_norm_backward_workspace_bytes.argtypes = [i64, i32, C.POINTER(C.c_size_t)]
        L.gad_layer_norm_backward.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i32, vp, vp, vp, i64, vp, vp, vp, C.c_size_t, vp]
        L.gad_class_loss_workspace_bytes.argtypes = [C.POINTER(_ClassLossArgs), C.POINTER(C.c_size_t)]
        L.gad_class_loss.argtypes = [C.POINTER(_ClassLossArgs), vp, C.c_size_t, vp]
        L.gad_policy_loss_workspace_bytes.argtypes = [C.POINTER(_PolicyLossArgs), C.POINTER(C.c_size_t)]
        L.gad_policy_loss.argtypes = [C.POINTER(_PolicyLossArgs), vp, C.c_size_t, vp]
        _DTYPES.update({torch.float32: 0, torch.float16: 1, torch.bfloat16: 2})
        _lib = L
    return _lib


def _matrix(t, name, device=None, shape=None):
    """Checks a row-major CUDA matrix; returns its row stride."""
    if t.dim() != 2 or t.dtype not in _DTYPES or not t.is_cuda:
        raise GadError(-1, "%s must be a float32, float16 or bfloat16 CUDA matrix" % name)
    if device is not None and t.device != device:
        raise GadError(-1, "%s is on another device" % name)
    if shape is not None and t.shape != shape:
        raise GadError(-1, "%s must be %d x %d" % ((name,) + shape))
    rows, cols = t.shape
    ld, inner = t.stride()
    if cols < 1 or (cols > 1 and inner != 1):
        raise GadError(-1, "%s must have at least one column, and its rows contiguous" % name)
    if cols > _MOST:
        raise GadError(-2, "%s has too many columns" % name)
    if rows <= 1:
        return max(ld, cols)
    if ld != 0 and ld < cols:
        raise GadError(-1, "the rows of %s overlap" % name)
    return ld


def _vector(t, name, n, dtypes, device):
    """Checks a contiguous CUDA vector of n elements (None passes); returns its address or None."""
    if t is None:
        return None
    if not (t.dtype in dtypes and t.device == device and t.shape == (n,) and t.is_contiguous()):
        raise GadError(-1, "%s must be a contiguous vector of %d elements (%s) on the same device" % (name, n, " or ".join(str(d) for d in dtypes)))
    return t.data_ptr()


@contextlib.contextmanager
def _switch(device, stream):
    """The tensors' device, and the stream asked for, made current: what is allocated then belongs to the stream that uses it."""
    with torch.cuda.device(device):
        if stream is None:
            yield
        else:
            if stream.device != device:
                raise GadError(-1, "the stream belongs to another device")
            with torch.cuda.stream(stream):
                yield


def _elsewhere(device, stream):
    return stream is not None or device.index != torch.cuda.current_device()


def _stream(device):
    """Address of torch's current stream (its object costs 2 us to make, a tenth of a small call)."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(device.index) if raw is not None else torch.cuda.current_stream(device).cuda_stream


def _ck(rc, what):
    if rc != GAD_OK:
        raise GadError(rc, what)


def layer_norm(x, gamma=None, beta=None, *, eps=1e-5, stream=None):
    """gad_layer_norm: ``(y, mean, rstd)`` of the rows of ``x`` [rows x cols]: y = (x - mean) * rstd * gamma + beta.

    x float32, float16 or bfloat16 with any row stride; gamma and beta [cols] in x's type or float32 (both in the same), or None.
    y has x's type and is contiguous; mean and rstd are float32 [rows] (``layer_norm_backward`` takes them).  Autograd does not see the call."""
    L = _load()
    ldx = _matrix(x, "x")
    rows, cols = x.shape
    dt, dev = x.dtype, x.device
    ptype = dt if gamma is None and beta is None else (gamma if gamma is not None else beta).dtype
    if ptype is not dt and ptype is not torch.float32:
        raise GadError(-1, "gamma and beta must have x's type or float32")
    g = _vector(gamma, "gamma", cols, (ptype,), dev)
    b = _vector(beta, "beta", cols, (ptype,), dev)
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return layer_norm(x, gamma, beta, eps=eps)
    y = torch.empty_like(x) if ldx == cols and not x.requires_grad else x.new_empty((rows, cols))     # (the former is the quicker)
    stats = x.new_empty((2, rows), dtype=torch.float32)
    at = stats.data_ptr()
    _ck(L.gad_layer_norm(x.data_ptr(), ldx, rows, cols, _DTYPES[dt], g, b, _DTYPES[ptype], eps, y.data_ptr(), cols, at, at + 4 * rows, _stream(dev)), "gad_layer_norm")
    mean, rstd = stats.unbind(0)
    return y, mean, rstd


@functools.lru_cache(maxsize=256)
def _norm_workspace(rows, cols):
    n = C.c_size_t(0)
    _ck(_load().gad_layer_norm_backward_workspace_bytes(rows, cols, C.byref(n)), "gad_layer_norm_backward_workspace_bytes")
    return n.value


def layer_norm_backward(dy, x, mean, rstd, gamma=None, *, param_grads=True, stream=None):
    """gad_layer_norm_backward: ``(dx, dgamma, dbeta)`` for the upstream gradient ``dy`` of ``layer_norm(x, gamma, beta)``.

    dx has x's type, dgamma and dbeta gamma's (x's without one); with ``param_grads=False`` they are None."""
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
    if _elsewhere(x.device, stream):
        with _switch(x.device, stream):
            return layer_norm_backward(dy, x, mean, rstd, gamma, param_grads=param_grads)
    dx = torch.empty_like(x) if ldx == cols and not x.requires_grad else x.new_empty((rows, cols))
    dgamma = dbeta = ws = None
    nbytes, at_g, at_b, at_ws = 0, None, None, None
    if param_grads:
        dgamma, dbeta = x.new_empty((2, cols), dtype=ptype).unbind(0)
        nbytes = _norm_workspace(rows, cols)
        ws = x.new_empty(nbytes, dtype=torch.uint8)
        at_g, at_b, at_ws = dgamma.data_ptr(), dbeta.data_ptr(), ws.data_ptr()
    _ck(L.gad_layer_norm_backward(dy.data_ptr(), lddy, x.data_ptr(), ldx, rows, cols, _DTYPES[x.dtype], g, _DTYPES[ptype], m, r, dx.data_ptr(), cols,
                                  at_g, at_b, at_ws, nbytes, _stream(x.device)), "gad_layer_norm_backward")
    return dx, dgamma, dbeta


class ClassLoss(NamedTuple):
    """What ``class_loss`` and ``distill_loss`` return.  ``loss`` float32 [1]; ``row_loss`` float32 [rows]; the gradients in the type of H,
    or None where not asked for; ``status`` int32 [1], zero unless a wait inside a kernel ran out."""
    loss: "object"
    row_loss: "object"
    dH: Optional["object"]
    dW: Optional["object"]
    db: Optional["object"]
    status: "object"

    def check(self):
        """Waits for the result; raises GAD_ERR_DEVICE_TIMEOUT if a bounded wait ran out, GAD_ERR_NONFINITE if the loss is not finite."""
        return _check_loss(self)


class PolicyLoss(NamedTuple):
    """What ``policy_loss`` returns: as ``ClassLoss``, and ``logp`` float32 [rows], the actions' log-probabilities (zero where a row does not count)."""
    loss: "object"
    row_loss: "object"
    logp: "object"
    dH: Optional["object"]
    dW: Optional["object"]
    db: Optional["object"]
    status: "object"

    def check(self):
        """Waits for the result; raises GAD_ERR_DEVICE_TIMEOUT if a bounded wait ran out, GAD_ERR_NONFINITE if the loss is not finite."""
        return _check_loss(self)


def _check_loss(r):
    code = int(r.status.item())
    if code:
        raise GadError(-7, "wait %d ran out" % code)
    if not bool(r.loss.isfinite().item()):
        raise GadError(-6, "the loss is not finite")
    return r


def _indices(t, name, shape, device):
    """Checks contiguous int32 / int64 indices; returns (address, bytes of one)."""
    if not (t.is_cuda and t.device == device and t.dtype in (torch.int32, torch.int64) and tuple(t.shape) == shape and t.is_contiguous()):
        raise GadError(-1, "%s must be a contiguous int32 or int64 tensor of shape %s on the same device" % (name, list(shape)))
    return t.data_ptr(), t.element_size()


def _class_loss(H, W, labels, classes, teacher, temperature, hard_weight, bias, row_weights, mean, scale, grads, stream, policy=None):
    """policy: None, or (old_logp, advantages, ref_logp, clip_low, clip_high, kl_weight)."""
    L = _load()
    ldh = _matrix(H, "H")
    N, D = H.shape
    dev, dt = H.device, H.dtype
    ldw = _matrix(W, "W", dev)
    V = W.shape[0]
    if W.dtype is not dt or W.shape[1] != D:
        raise GadError(-1, "W must have H's type and number of columns")
    if V < 1 or (V > 1 and ldw == 0):
        raise GadError(-1, "W must have a row for every class")
    if V > _MOST:
        raise GadError(-2, "W has too many rows")
    b = _vector(bias, "bias", V, (dt,), dev)
    w = _vector(row_weights, "row_weights", N, (torch.float32,), dev)
    lab, lab_bytes = _indices(labels, "labels", (N,), dev) if labels is not None else (None, 4)
    k, tc, tc_bytes, te, te_type = 0, None, 4, None, 0
    if classes is not None:
        if classes.dim() != 2 or classes.shape[1] < 1:
            raise GadError(-1, "classes must be rows x k, k of 1 and more")
        k = classes.shape[1]
        if k > _MOST:
            raise GadError(-2, "classes has too many slots")
        tc, tc_bytes = _indices(classes, "classes", (N, k), dev)
        if not (teacher.is_cuda and teacher.device == dev and teacher.dtype in _DTYPES and tuple(teacher.shape) == (N, k) and teacher.is_contiguous()):
            raise GadError(-1, "teacher must be a contiguous floating tensor of the shape of classes on the same device")
        te, te_type = teacher.data_ptr(), _DTYPES[teacher.dtype]
    if policy is not None:
        of_rows = [_vector(t, name, N, (torch.float32,), dev) for t, name in zip(policy[:3], ("old_logp", "advantages", "ref_logp"))]
    want = {"H", "W", "b"} if grads is True else set() if not grads else set(grads)
    if not want <= {"H", "W", "b"}:
        raise GadError(-1, "grads is True, False or some of H, W and b")
    if _elsewhere(dev, stream):
        with _switch(dev, stream):
            return _class_loss(H, W, labels, classes, teacher, temperature, hard_weight, bias, row_weights, mean, scale, grads, None, policy)
    out = H.new_empty(N + 1 if policy is None else 2 * N + 1, dtype=torch.float32)
    status = H.new_empty(1, dtype=torch.int32)
    dH = H.new_empty((N, D)) if "H" in want else None
    dW = W.new_empty((V, D)) if "W" in want else None
    db = W.new_empty(V) if "b" in want and b is not None else None
    at = out.data_ptr()
    a = _ClassLossArgs(_DTYPES[dt], D, V, N, H.data_ptr(), ldh, W.data_ptr(), ldw, b, lab, lab_bytes, k, tc, tc_bytes, te_type, te, temperature,
                       hard_weight, w, scale, 1 if mean else 0, at + 4 * N, at, dH.data_ptr() if dH is not None else None, D,
                       dW.data_ptr() if dW is not None else None, D, db.data_ptr() if db is not None else None, status.data_ptr())
    nbytes = C.c_size_t(0)
    if policy is not None:
        a = _PolicyLossArgs(a, *of_rows, *policy[3:], at + 4 * (N + 1))
        _ck(L.gad_policy_loss_workspace_bytes(C.byref(a), C.byref(nbytes)), "gad_policy_loss")
        ws = H.new_empty(nbytes.value, dtype=torch.uint8)
        _ck(L.gad_policy_loss(C.byref(a), ws.data_ptr(), nbytes.value, _stream(dev)), "gad_policy_loss")
        return PolicyLoss(out[N:N + 1], out[:N], out[N + 1:], dH, dW, db, status)
    _ck(L.gad_class_loss_workspace_bytes(C.byref(a), C.byref(nbytes)), "gad_class_loss")
    ws = H.new_empty(nbytes.value, dtype=torch.uint8)     # (torch's blocks start on 512 bytes)
    _ck(L.gad_class_loss(C.byref(a), ws.data_ptr(), nbytes.value, _stream(dev)), "gad_class_loss")
    return ClassLoss(out[N:], out[:N], dH, dW, db, status)


def class_loss(H, W, labels, *, bias=None, row_weights=None, mean=True, scale=1.0, grads=True, stream=None):
    """gad_class_loss with labels: softmax cross entropy of the output layer z = H W^T + bias over many classes.  Of z a block of about 2 GB at
    most is held at a time for gradients (2 bytes a logit in the 16-bit types, 10 in float32), and none without.

    H [rows x cols] and W [classes x cols] float32, float16 or bfloat16 (both the same), any row stride; labels int32 / int64 [rows], below
    zero: the row does not count; bias [classes] in the same type, -inf takes a class out.
    loss = scale * sum_i row_weights_i row_loss_i, with ``mean`` divided by the number of rows that count.
    grads: True, False, or some of "H", "W", "b" as a string or set.  Returns a ``ClassLoss``; autograd does not see the call."""
    if labels is None:
        raise GadError(-1, "labels are needed")
    return _class_loss(H, W, labels, None, None, 1.0, 1.0, bias, row_weights, mean, scale, grads, stream)


def distill_loss(H, W, classes, teacher, *, temperature=1.0, labels=None, hard_weight=0.0, bias=None, row_weights=None, mean=True, scale=1.0,
                 grads=True, stream=None):
    """gad_class_loss with a teacher: classes int32 / int64 [rows x k] (below zero: the slot is unused) and its logits there, ``teacher``
    [rows x k] of any of the three types, k of 1 to 1024.  With q = softmax(teacher / T) over the used slots of a row and z as in ``class_loss``,
    row_loss = (1 - hard_weight) T^2 sum q (log q - log softmax(z / T)) + hard_weight * cross entropy against ``labels`` (where given)."""
    if classes is None or teacher is None:
        raise GadError(-1, "classes and teacher are needed")
    return _class_loss(H, W, labels, classes, teacher, temperature, hard_weight if labels is not None else 0.0, bias, row_weights, mean, scale, grads, stream)


def policy_loss(H, W, actions, old_logp, advantages, *, ref_logp=None, clip=0.2, kl_weight=0.0, bias=None, row_weights=None, mean=True, scale=1.0, grads=True, stream=None):
    """gad_policy_loss: the clipped policy loss of actions chosen among the classes of z = H W^T + bias, with a KL term towards a reference policy.

    With lp the log-probability of a row's action and r = exp(lp - old_logp), row_loss = -min(r A, clip(r, 1 - low, 1 + high) A) + kl_weight (exp(ref_logp - lp) -
    (ref_logp - lp) - 1).  actions as ``class_loss``'s labels (below zero: the row does not count); old_logp, advantages and ref_logp float32 [rows] (without ref_logp there is no
    KL term); clip: one number, or (low, high) with high up to infinity.  Everything else as in ``class_loss``.  Returns a ``PolicyLoss``, whose ``logp`` a later call may be given as
    ``old_logp``; for the log-probabilities alone: ``-class_loss(H, W, actions, grads=False).row_loss`` (its sums are cut otherwise: the last bits may differ)."""
    if actions is None or old_logp is None or advantages is None:
        raise GadError(-1, "actions, old_logp and advantages are needed")
    if isinstance(clip, (tuple, list)) and len(clip) != 2:
        raise GadError(-1, "clip is one number, or (low, high)")
    low, high = clip if isinstance(clip, (tuple, list)) else (clip, clip)
    return _class_loss(H, W, actions, None, None, 1.0, 1.0, bias, row_weights, mean, scale, grads, stream, (old_logp, advantages, ref_logp, low, high, kl_weight))
