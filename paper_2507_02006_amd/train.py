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


def _dtype(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.float32: B_.DTYPE_F32, torch.bfloat16: B_.DTYPE_BF16, torch.float16: B_.DTYPE_F16})
    d = _DTYPES.get(t)
    if d is None:
        raise TypeError("expected float32, bfloat16 or float16, got %s" % (t,))
    return d


def _dense(x, name: str) -> B_.Dense:
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError("%s must be a device matrix" % name)
    m, n = x.shape
    ld = x.stride(0) if m > 1 else n
    if (n > 1 and x.stride(1) != 1) or (m > 1 and ld < n):
        raise ValueError("%s needs unit column stride and rows that do not overlap" % name)
    return B_.Dense(m, n, ld, _dtype(x.dtype), 0, x.data_ptr())


def _vector(x, n: int, name: str, dtype=None) -> int:
    """Address of a contiguous device vector of n values."""
    if x.dim() != 1 or x.shape[0] != n or not x.is_cuda or (n > 1 and x.stride(0) != 1):
        raise ValueError("%s must be a contiguous device vector of %d values" % (name, n))
    if dtype is not None and x.dtype != dtype:
        raise TypeError("%s must be %s" % (name, dtype))
    return x.data_ptr()


def _same_device(first, *others) -> None:
    for x in others:
        if x is not None and x.device != first.device:
            raise ValueError("tensors on %s and %s" % (first.device, x.device))


@contextlib.contextmanager
def _other_stream(device, stream):
    import torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield stream.cuda_stream


@contextlib.contextmanager
def _current(device):
    import torch
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


def _on(x, stream):
    """Context in which allocations belong to ``stream`` on x's device; gives
    the hipStream_t."""
    import torch
    if stream is not None:
        return _other_stream(x.device, stream)
    if x.device.index == torch.cuda.current_device():
        return _Here(torch.cuda.current_stream(x.device).cuda_stream)
    return _current(x.device)


def layer_norm(X, gamma=None, beta=None, *, eps: float = 1e-5, out_dtype=None, stats: bool = True, out=None,
               stream=None):
    """Layer norm of the rows of X (aires_layer_norm): Y = (X - mean) * rstd *
    gamma + beta.  gamma, beta: vectors of one type, or None.  Y has
    ``out_dtype`` (X's type by default) unless ``out`` is given.  Returns
    (Y, mean, rstd); mean and rstd (float32, for ``layer_norm_backward``)
    are None when ``stats`` is false."""
    import torch
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
            out = torch.empty((m, n), dtype=out_dtype or X.dtype, device=X.device)
        elif out_dtype is not None and out.dtype != out_dtype:
            raise TypeError("out is %s, out_dtype %s" % (out.dtype, out_dtype))
        dy = _dense(out, "out")
        st = torch.empty((2, m), dtype=torch.float32, device=X.device) if stats else None
        at = st.data_ptr() if stats else 0
        B_.check(B_.load().aires_layer_norm(ctypes.byref(dx), g, b, _dtype(w.dtype) if w is not None else 0, eps,
                                            ctypes.byref(dy), at or None, at + 4 * m if at else None, s),
                 "aires_layer_norm")
    return (out, st[0], st[1]) if stats else (out, None, None)


def layer_norm_backward(dY, X, mean, rstd, gamma=None, *, need_dx: bool = True, need_weights: bool = True,
                        dx_dtype=None, stream=None):
    """Gradients of ``layer_norm`` (aires_layer_norm_backward) from dY, X and
    the statistics that the forward call returned.  Returns (dX, dgamma,
    dbeta): dX of ``dx_dtype`` (X's type by default), dgamma and dbeta of
    gamma's type (float32 without gamma); None where not needed."""
    import torch
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
        out = torch.empty((m, n), dtype=dx_dtype or X.dtype, device=X.device) if need_dx else None
        dg = db = work = None
        need = ctypes.c_int64(0)
        if need_weights:
            B_.check(lib.aires_layer_norm_workspace(m, n, ctypes.byref(need)), "aires_layer_norm_workspace")
            dg, db = torch.empty(n, dtype=wt, device=X.device), torch.empty(n, dtype=wt, device=X.device)
            work = torch.empty(need.value, dtype=torch.uint8, device=X.device)
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
    import torch
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
        work = torch.empty(need.value, dtype=torch.uint8, device=H.device)
        loss = torch.empty((), dtype=torch.float32, device=H.device)
        rows = torch.empty(t, dtype=torch.float32, device=H.device)
        dH = torch.empty((t, d), dtype=H.dtype, device=H.device) if grads else None
        dW = torch.empty((v, d), dtype=W.dtype, device=H.device) if grads else None
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
    import torch
    if bits == 32:
        return tuple([torch.zeros_like(p, dtype=torch.float32) for p in params] for _ in range(2))
    if bits != 8:
        raise ValueError("bits must be 8 or 32")
    return tuple([(torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(kind),
                   torch.zeros(-(-p.numel() // B_.ADAMW_BLOCK), dtype=torch.float32, device=p.device))
                  for p in params] for kind in (torch.float8_e4m3fn, torch.float8_e5m2))


def _moment(x, p, kind):
    """(address, address of the scales) of one moment of parameter p."""
    import torch
    if isinstance(x, tuple):
        codes, scales = x
        if codes.dtype != kind or codes.shape != p.shape or not codes.is_contiguous() or codes.device != p.device:
            raise ValueError("expected contiguous %s codes of the parameter's shape" % kind)
        if scales.dtype != torch.float32 or scales.numel() != -(-p.numel() // B_.ADAMW_BLOCK) or \
                not scales.is_contiguous() or scales.device != p.device:
            raise ValueError("expected one float32 scale for each %d values" % B_.ADAMW_BLOCK)
        return codes.data_ptr(), scales.data_ptr()
    if x.dtype != torch.float32 or x.shape != p.shape or not x.is_contiguous() or x.device != p.device:
        raise ValueError("expected a contiguous float32 moment of the parameter's shape")
    return x.data_ptr(), None


def adamw(params, grads, exp_avg, exp_avg_sq, *, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
          weight_decay: float = 0.01, grad_scale: float = 1.0, seed: int = 0, copies=None, stream=None) -> None:
    """One AdamW step over lists of tensors, in place (aires_adamw).  params:
    contiguous float32, bfloat16 or float16; grads: of any of these types;
    exp_avg, exp_avg_sq: as from ``adamw_state``, in 32 or 8 bits (``seed``
    then drives their rounding: pass another one each step); copies:
    tensors that receive the updated parameters in their own type (or None,
    also for single entries).  ``step`` counts from 1."""
    import torch
    n = len(params)
    if not (len(grads) == len(exp_avg) == len(exp_avg_sq) == n) or (copies is not None and len(copies) != n):
        raise ValueError("params, grads, moments and copies differ in number")
    if n == 0:
        return
    table = (B_.AdamWTensor * n)()
    device = params[0].device
    for k, p in enumerate(params):
        g = grads[k]
        if g.shape != p.shape or not p.is_contiguous() or not g.is_contiguous():
            raise ValueError("parameter %d and its gradient must be contiguous and of one shape" % k)
        if not p.is_cuda or p.device != device or g.device != device:
            raise ValueError("all tensors must be on one device")
        m, ms = _moment(exp_avg[k], p, torch.float8_e4m3fn)
        v, vs = _moment(exp_avg_sq[k], p, torch.float8_e5m2)
        c = copies[k] if copies is not None else None
        if c is not None and (c.shape != p.shape or not c.is_contiguous() or c.device != device):
            raise ValueError("copy %d must be contiguous and of its parameter's shape" % k)
        table[k] = (p.numel(), p.data_ptr(), g.data_ptr(), m, v, ms, vs, c.data_ptr() if c is not None else None,
                    _dtype(p.dtype), _dtype(g.dtype), _dtype(c.dtype) if c is not None else 0, 0)
    o = B_.AdamWOpts(ctypes.sizeof(B_.AdamWOpts), int(seed) & 0xFFFFFFFF, int(step), lr, betas[0], betas[1], eps,
                     weight_decay, grad_scale)
    with _on(params[0], stream) as s:
        B_.check(B_.load().aires_adamw(table, n, ctypes.byref(o), s), "aires_adamw")
