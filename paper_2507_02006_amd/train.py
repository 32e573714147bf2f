"""Training on aggregated features: layer norm, softmax cross entropy against
a table, AdamW (the dense-array calls of include/aires.h; argument
marshalling only).

Matrices are device torch tensors of float32, bfloat16 or float16 with unit
column stride (any row stride).  Work is enqueued on ``stream`` (torch's
current stream by default), where inputs must be ready; outputs and
workspaces are allocated for that stream and valid once it reaches the
enqueued kernels.
"""
from __future__ import annotations

import contextlib
import ctypes
from dataclasses import dataclass
from typing import Any

from . import _binding as B_

_DTYPES: dict = {}
_torch = None


def _load_torch():
    """torch, imported with the first call (the package itself does not)."""
    global _torch
    import torch
    _torch = torch
    return torch


def _dtype(t) -> int:
    d = _DTYPES.get(t)
    if d is None:
        torch = _torch or _load_torch()
        _DTYPES.update({torch.float32: B_.DTYPE_F32, torch.bfloat16: B_.DTYPE_BF16, torch.float16: B_.DTYPE_F16})
        d = _DTYPES.get(t)
        if d is None:
            raise TypeError("expected float32, bfloat16 or float16, got %s" % (t,))
    return d


def _dense(x, name: str) -> B_.Dense:
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError("%s must be a device matrix" % name)
    m, n = x.shape
    ld = n
    if not x.is_contiguous():
        if m > 1:
            ld = x.stride(0)
        if (n > 1 and x.stride(1) != 1) or (m > 1 and ld < n):
            raise ValueError("%s needs unit column stride and rows that do not overlap" % name)
    return B_.Dense(m, n, ld, _dtype(x.dtype), 0, x.data_ptr())


def _vector(x, n: int, name: str, dtype=None) -> int:
    """Address of a contiguous device vector of n values."""
    if x.dim() != 1 or x.shape[0] != n or not x.is_cuda or not x.is_contiguous():
        raise ValueError("%s must be a contiguous device vector of %d values" % (name, n))
    if dtype is not None and x.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    return x.data_ptr()


def _same_device(first, *others) -> None:
    d = first.get_device()
    for x in others:
        if x is not None and x.get_device() != d:
            raise ValueError("tensors on %s and %s" % (first.device, x.device))


@contextlib.contextmanager
def _other_stream(device, stream):
    torch = _torch or _load_torch()
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield stream.cuda_stream


@contextlib.contextmanager
def _current(device):
    torch = _torch or _load_torch()
    with torch.cuda.device(device):
        yield torch.cuda.current_stream(device).cuda_stream


class _Here:
    """The current stream of the current device: the usual case, without the
    cost of switching."""
    __slots__ = ("handle",)

    def __init__(self, handle):
        self.handle = handle

    def __enter__(self):
        return self.handle

    def __exit__(self, *a):
        return False


def _raw_stream(device: int) -> int:
    """hipStream_t of the device's current stream (0.1 us where torch hands
    out the handle itself, 2 us through a stream object)."""
    torch = _torch or _load_torch()
    f = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return f(device) if f is not None else torch.cuda.current_stream(device).cuda_stream


def _on(x, stream):
    """Context in which allocations belong to ``stream`` on x's device; gives
    the hipStream_t."""
    torch = _torch or _load_torch()
    if stream is not None:
        return _other_stream(x.device, stream)
    d = x.get_device()
    if d == torch.cuda.current_device():
        return _Here(_raw_stream(d))
    return _current(x.device)


def layer_norm(X, gamma=None, beta=None, *, eps: float = 1e-5, out_dtype=None, stats: bool = True, out=None,
               stream=None):
    """Layer norm of the rows of X (aires_layer_norm): Y = (X - mean) * rstd *
    gamma + beta.  gamma, beta: vectors of one type, or None.  Y has
    ``out_dtype`` (X's type by default) unless ``out`` is given.  Returns
    (Y, mean, rstd); mean and rstd (float32, for ``layer_norm_backward``)
    are None when ``stats`` is false."""
    torch = _torch or _load_torch()
    dx = _dense(X, "X")
    m, n = X.shape
    if gamma is not None and beta is not None and gamma.dtype != beta.dtype:
        raise TypeError("gamma and beta have different types")
    w = gamma if gamma is not None else beta
    g = _vector(gamma, n, "gamma") if gamma is not None else None
    b = _vector(beta, n, "beta") if beta is not None else None
    _same_device(X, gamma, beta, out)
    with _on(X, stream) as s:
        if out is None:
            out = X.new_empty((m, n), dtype=out_dtype)
        elif out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out is %s, out_dtype %s" % (out.dtype, out_dtype))
        dy = _dense(out, "out")
        st = X.new_empty((2, m), dtype=torch.float32) if stats else None
        at = st.data_ptr() if stats else 0
        B_.check(B_.load().aires_layer_norm(ctypes.byref(dx), g, b, _dtype(w.dtype) if w is not None else 0, eps,
                                            ctypes.byref(dy), at or None, at + 4 * m if at else None, s),
                 "aires_layer_norm")
    return (out, *st.unbind()) if stats else (out, None, None)


def layer_norm_backward(dY, X, mean, rstd, gamma=None, *, need_dx: bool = True, need_weights: bool = True,
                        dx_dtype=None, stream=None):
    """Gradients of ``layer_norm`` (aires_layer_norm_backward) from dY, X and
    the statistics that the forward call returned.  Returns (dX, dgamma,
    dbeta): dX of ``dx_dtype`` (X's type by default), dgamma and dbeta of
    gamma's type (float32 without gamma); None where not needed."""
    torch = _torch or _load_torch()
    dy, dx = _dense(dY, "dY"), _dense(X, "X")
    m, n = X.shape
    if tuple(dY.shape) != (m, n):
        raise ValueError("dY is %s, X %s" % (tuple(dY.shape), (m, n)))
    g = _vector(gamma, n, "gamma") if gamma is not None else None
    mu, r = _vector(mean, m, "mean", torch.float32), _vector(rstd, m, "rstd", torch.float32)
    _same_device(X, dY, gamma, mean, rstd)
    lib = B_.load()
    with _on(X, stream) as s:
        wt = gamma.dtype if gamma is not None else torch.float32
        out = X.new_empty((m, n), dtype=dx_dtype) if need_dx else None
        dg = db = work = None
        need = ctypes.c_int64(0)
        if need_weights:
            B_.check(lib.aires_layer_norm_workspace(m, n, ctypes.byref(need)), "aires_layer_norm_workspace")
            dg, db = X.new_empty((2, n), dtype=wt).unbind()
            work = X.new_empty(need.value, dtype=torch.uint8)
        B_.check(lib.aires_layer_norm_backward(
            ctypes.byref(dy), ctypes.byref(dx), mu, r, g, _dtype(wt), ctypes.byref(_dense(out, "dX")) if need_dx else None,
            dg.data_ptr() if need_weights else None, db.data_ptr() if need_weights else None,
            work.data_ptr() if need_weights else None, need.value, s), "aires_layer_norm_backward")
    return out, dg, db


@dataclass
class Xent:
    """What ``linear_xent`` returns: loss (a float32 scalar tensor), row_loss
    (float32, one per row), dH and dW (None without gradients)."""
    loss: Any
    row_loss: Any
    dH: Any = None
    dW: Any = None


def linear_xent(H, W, labels, *, reduction: str = "mean", grads: bool = True, grad_scale: float = 1.0,
                stream=None) -> Xent:
    """Softmax cross entropy of the scores H W^T against labels, and its
    gradients, without storing the scores (aires_linear_xent).  H: (t x d)
    features; W: (v x d), one row per class or table entry, of H's type;
    labels: t integers (int32 or int64), a label outside [0, v) marks a row
    without a target.  reduction: "mean" over labelled rows or "sum".  dH and
    dW (of H's and W's type) are multiplied with ``grad_scale``."""
    torch = _torch or _load_torch()
    if reduction not in ("mean", "sum"):
        raise ValueError("reduction must be 'mean' or 'sum'")
    if labels.dtype not in (torch.int32, torch.int64):
        raise TypeError("labels must be int32 or int64")
    h, w = _dense(H, "H"), _dense(W, "W")
    t, d = H.shape
    v = W.shape[0]
    if W.shape[1] != d or W.dtype != H.dtype:
        raise ValueError("H is %s of %s, W %s of %s" % ((t, d), H.dtype, tuple(W.shape), W.dtype))
    y = _vector(labels, t, "labels")
    _same_device(H, W, labels)
    lib = B_.load()
    with _on(H, stream) as s:
        need = ctypes.c_int64(0)
        B_.check(lib.aires_linear_xent_workspace(t, d, v, h.dtype, int(grads), ctypes.byref(need)),
                 "aires_linear_xent_workspace")
        work = H.new_empty(need.value, dtype=torch.uint8)
        loss = H.new_empty((), dtype=torch.float32)
        rows = H.new_empty(t, dtype=torch.float32)
        dH = H.new_empty((t, d)) if grads else None
        dW = H.new_empty((v, d)) if grads else None
        B_.check(lib.aires_linear_xent(
            ctypes.byref(h), ctypes.byref(w), y, int(labels.dtype == torch.int64),
            B_.REDUCE_MEAN if reduction == "mean" else B_.REDUCE_SUM, grad_scale, loss.data_ptr(), rows.data_ptr(),
            ctypes.byref(_dense(dH, "dH")) if grads else None, ctypes.byref(_dense(dW, "dW")) if grads else None,
            work.data_ptr(), need.value, s), "aires_linear_xent")
    return Xent(loss, rows, dH, dW)


def adamw_state(params, bits: int = 32):
    """Zero moments for ``adamw``: two lists, one entry per parameter.  32
    bits: float32 tensors.  8 bits: (codes, scales) pairs, codes of the
    parameter's shape in float8_e4m3fn (first moment) and float8_e5m2 (second),
    one float32 scale for each 256 values."""
    torch = _torch or _load_torch()
    if bits == 32:
        return tuple([torch.zeros_like(p, dtype=torch.float32) for p in params] for _ in range(2))
    if bits != 8:
        raise ValueError("bits must be 8 or 32")
    return tuple([(torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(kind),
                   torch.zeros(-(-p.numel() // B_.ADAMW_BLOCK), dtype=torch.float32, device=p.device))
                  for p in params] for kind in (torch.float8_e4m3fn, torch.float8_e5m2))


def _codes(x, p, kind):
    """(address, address of the scales) of an 8-bit moment of parameter p."""
    torch = _torch or _load_torch()
    codes, scales = x
    if codes.dtype != kind or codes.shape != p.shape or not codes.is_contiguous():
        raise ValueError("expected contiguous %s codes of the parameter's shape" % kind)
    if scales.dtype != torch.float32 or scales.numel() != -(-p.numel() // B_.ADAMW_BLOCK) or not scales.is_contiguous():
        raise ValueError("expected one float32 scale for each %d values" % B_.ADAMW_BLOCK)
    if not codes.get_device() == scales.get_device() == p.get_device():
        raise ValueError("all tensors must be on one device")
    return codes.data_ptr(), scales.data_ptr()


def adamw(params, grads, exp_avg, exp_avg_sq, *, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
          weight_decay: float = 0.01, grad_scale: float = 1.0, seed: int = 0, copies=None, stream=None) -> None:
    """One AdamW step over lists of tensors, in place (aires_adamw).  params:
    contiguous float32, bfloat16 or float16; grads: of any of these types;
    exp_avg, exp_avg_sq: as from ``adamw_state``, in 32 or 8 bits (``seed``
    then drives their rounding: pass another one each step); copies:
    tensors that receive the updated parameters in their own type (or None,
    also for single entries).  ``step`` counts from 1."""
    torch = _torch or _load_torch()
    n = len(params)
    if not (len(grads) == len(exp_avg) == len(exp_avg_sq) == n) or (copies is not None and len(copies) != n):
        raise ValueError("params, grads, moments and copies differ in number")
    if n == 0:
        return
    f32 = torch.float32
    device = params[0].get_device()
    if device < 0:
        raise ValueError("parameters must be on a device")
    rows = []  # the tensors' descriptors, ten 64-bit words each
    for p, g, m, v, c in zip(params, grads, exp_avg, exp_avg_sq, copies or (None,) * n):
        shape = p.shape
        if g.shape != shape or not p.is_contiguous() or not g.is_contiguous():
            raise ValueError("a parameter and its gradient must be contiguous and of one shape")
        if p.get_device() != device or g.get_device() != device:
            raise ValueError("all tensors must be on one device")
        ms = vs = cp = ct = 0
        if isinstance(m, tuple):
            m, ms = _codes(m, p, torch.float8_e4m3fn)
            v, vs = _codes(v, p, torch.float8_e5m2)
        else:
            for x in (m, v):
                if x.dtype != f32 or x.shape != shape or not x.is_contiguous() or x.get_device() != device:
                    raise ValueError("expected contiguous float32 moments of the parameter's shape")
            m, v = m.data_ptr(), v.data_ptr()
        if c is not None:
            if c.shape != shape or not c.is_contiguous() or c.get_device() != device:
                raise ValueError("a copy must be contiguous and of its parameter's shape")
            cp, ct = c.data_ptr(), _dtype(c.dtype)
        rows += (p.numel(), p.data_ptr(), g.data_ptr(), m, v, ms, vs, cp, _dtype(p.dtype) | _dtype(g.dtype) << 32, ct)
    table = (ctypes.c_int64 * (10 * n))(*rows)
    o = B_.AdamWOpts(ctypes.sizeof(B_.AdamWOpts), int(seed) & 0xFFFFFFFF, int(step), lr, betas[0], betas[1], eps,
                     weight_decay, grad_scale)
    with _on(params[0], stream) as s:
        B_.check(B_.load().aires_adamw(ctypes.addressof(table), n, ctypes.byref(o), s), "aires_adamw")
