"""Training on aggregated features: layer norm, softmax cross entropy against
a table, AdamW (the dense-array calls of include/aires.h; argument
marshalling only).

Matrices are device torch tensors of float32, bfloat16 or float16 with unit
column stride (any row stride).  The calls take no part in autograd: gradients
are asked for by their own calls, and tensors that are written count a version.
Work is enqueued on ``stream`` (torch's
current stream by default), where inputs must be ready; outputs and
workspaces are allocated for that stream and valid once it reaches the
enqueued kernels.  Tensors given to a call with ``stream`` may be released
before that: their memory is not reused until then.
"""
from __future__ import annotations

import contextlib
import importlib.machinery
import importlib.util
import os
from dataclasses import dataclass
from typing import Any

from . import _binding as B_

_torch = None
_calls = None
CALLS_PATH = os.path.join(B_.HERE, "_calls.so")


def _load():
    """torch and the compiled calls, loaded with the first call (the package
    itself does not import torch).  There is no fallback path."""
    global _torch, _calls
    import torch
    lib = B_.load()
    if not os.path.exists(CALLS_PATH):
        raise RuntimeError("_calls.so is not built (run __graft_entry__.build()); there is no fallback path")
    loader = importlib.machinery.ExtensionFileLoader("_calls", CALLS_PATH)
    spec = importlib.util.spec_from_file_location("_calls", CALLS_PATH, loader=loader)
    m = importlib.util.module_from_spec(spec)
    loader.exec_module(m)
    if m.abi_version() != lib.aires_abi_version():
        raise RuntimeError("_calls.so is linked to another libaires.so (rebuild it)")
    m.set_error(B_.AiresError)
    _torch, _calls = torch, m
    return m


@contextlib.contextmanager
def _other_stream(device, stream):
    torch = _torch
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
    with torch.cuda.device(device), torch.cuda.stream(stream):
        yield stream.cuda_stream


@contextlib.contextmanager
def _current(device):
    torch = _torch
    with torch.cuda.device(device):
        yield torch.cuda.current_stream(device).cuda_stream


def _here(x):
    """hipStream_t of the current stream if x is on the current device, the
    usual case, which needs no switching; else None."""
    d = x.get_device()
    if d < 0:
        raise ValueError("expected device tensors")
    if d != _torch.cuda.current_device():
        return None
    raw = getattr(_torch._C, "_cuda_getCurrentRawStream", None)  # (a stream object costs 2 us)
    return raw(d) if raw is not None else _torch.cuda.current_stream(d).cuda_stream


def _run(call, x, stream, *args):
    """call(*args, hipStream_t) where allocations belong to ``stream`` (None:
    the current one) on x's device."""
    if stream is None:
        s = _here(x)
        if s is not None:
            return call(*args, s)
        with _current(x.device) as s:
            return call(*args, s)
    if x.get_device() < 0:
        raise ValueError("expected device tensors")
    with _other_stream(x.device, stream) as s:
        _keep(args, _torch.cuda.current_stream(x.device))
        return call(*args, s)


def _keep(args, stream):
    """Tells torch's allocator that the tensors in ``args`` (sequences and pairs
    of them too) are in use on ``stream``, which may not be the one that they
    were made on."""
    for x in args:
        if isinstance(x, _torch.Tensor):
            if x.is_cuda:
                x.record_stream(stream)
        elif hasattr(x, "__getitem__"):
            _keep(x, stream)


def layer_norm(X, gamma=None, beta=None, *, eps: float = 1e-5, out_dtype=None, stats: bool = True, out=None,
               stream=None):
    """Layer norm of the rows of X (aires_layer_norm): Y = (X - mean) * rstd *
    gamma + beta.  gamma, beta: vectors of one type, or None.  Y has
    ``out_dtype`` (X's type by default) unless ``out`` is given.  Returns
    (Y, mean, rstd); mean and rstd (float32, for ``layer_norm_backward``)
    are None when ``stats`` is false."""
    c = _calls or _load()
    return _run(c.layer_norm, X, stream, X, gamma, beta, eps, out_dtype, stats, out)


def layer_norm_backward(dY, X, mean, rstd, gamma=None, *, need_dx: bool = True, need_weights: bool = True,
                        dx_dtype=None, stream=None):
    """Gradients of ``layer_norm`` (aires_layer_norm_backward) from dY, X and
    the statistics that the forward call returned.  Returns (dX, dgamma,
    dbeta): dX of ``dx_dtype`` (X's type by default), dgamma and dbeta of
    gamma's type (float32 without gamma); None where not needed."""
    c = _calls or _load()
    return _run(c.layer_norm_backward, X, stream, dY, X, mean, rstd, gamma, need_dx, need_weights, dx_dtype)


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
    if reduction not in ("mean", "sum"):
        raise ValueError("reduction must be 'mean' or 'sum'")
    c = _calls or _load()
    return Xent(*_run(c.linear_xent, H, stream, H, W, labels, reduction == "mean", grads, grad_scale))


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


def adamw(params, grads, exp_avg, exp_avg_sq, *, step: int, lr: float, betas=(0.9, 0.999), eps: float = 1e-8,
          weight_decay: float = 0.01, grad_scale=1.0, seed: int = 0, copies=None, stream=None) -> None:
    """One AdamW step over lists of tensors, in place (aires_adamw).  params:
    contiguous float32, bfloat16 or float16; grads: of any of these types;
    exp_avg, exp_avg_sq: as from ``adamw_state``, in 32 or 8 bits (``seed``
    then drives their rounding: pass another one each step); copies:
    tensors that receive the updated parameters in their own type (or None,
    also for single entries).  ``grad_scale``: a number, or a float32 scalar on
    the device (as ``grad_norm`` returns), which the kernels read; another tensor
    of one value is read now, which waits for the device if it is there.  With a
    factor of 0 on the device all gradients count 0, infinite ones too; with one
    that is not finite the step is left out.  ``step`` counts from 1.  A graph that captured the call repeats its step, options and
    seed."""
    c = _calls or _load()
    if len(params) == 0 and len(grads) == len(exp_avg) == len(exp_avg_sq) == 0:
        return
    if len(params) == 0:
        raise ValueError("params, grads, moments and copies differ in number")
    _run(c.adamw, params[0], stream, params, grads, exp_avg, exp_avg_sq, copies, step, lr, betas[0], betas[1], eps,
         weight_decay, grad_scale, int(seed) & 0xFFFFFFFF)
