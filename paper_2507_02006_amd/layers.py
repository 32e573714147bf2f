"""Layers on top of the aggregated features: a norm with a residual stream,
matrices held in 8 bits and their product, log probabilities of classes, and
the norm of all gradients (the calls of include/aires.h that follow the training
calls; argument marshalling only).

The rules of the training calls (train.py) hold: device torch tensors of float32,
bfloat16 or float16 with unit column stride, no part in autograd, work enqueued
on ``stream`` (torch's current stream by default), tensors that are written count a
version.  A matrix held in 8 bits is a pair (codes, scales): codes in
float8_e4m3fn, and one float32 scale for each 128 columns of a row (scales: rows
x ceil(columns / 128)) or of 128 rows ("tiles": ceil(rows / 128) x ceil(columns /
128)).
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Any

from . import train as T


def _call():
    return T._calls or T._load()


def rms_norm(X, gamma=None, *, residual=None, eps: float = 1e-6, out_dtype=None, stats: bool = True, out=None,
             sum_out=None, stream=None):
    """Root-mean-square norm of the rows of S = X + residual (of X without one)
    (aires_rms_norm): Y = S * rstd * gamma, the norm being that of S as it is
    stored.  Y has ``out_dtype`` (X's type by default; torch.float8_e4m3fn: a
    pair (codes, scales)) unless ``out`` is given; S has residual's type unless
    ``sum_out`` is given, which may be ``residual`` or X itself.  Returns (Y, S,
    rstd); S is None without a residual, rstd (float32, for
    ``rms_norm_backward``) when ``stats`` is false."""
    return T._run(_call().rms_norm, X, stream, X, gamma, residual, eps, out_dtype, stats, out, sum_out)


def rms_norm_backward(dY, S, rstd, gamma=None, *, dS=None, need_dx: bool = True, need_weights: bool = True,
                      dx_dtype=None, stream=None):
    """Gradients of ``rms_norm`` (aires_rms_norm_backward) from dY, the rows that
    were normalised (S, or X without a residual) and rstd.  dS: the gradient that
    reaches S past the norm, or None.  Returns (dX, dgamma): dX, the gradient of
    X and of the residual alike, of ``dx_dtype`` (S's type by default), dgamma of
    gamma's type (float32 without gamma); None where not needed."""
    return T._run(_call().rms_norm_backward, S, stream, dY, S, rstd, gamma, dS, need_dx, need_weights, dx_dtype)


def quantize_8bit(X, *, tiles: bool = False, order: str = "rows", stream=None):
    """X held in 8 bits (aires_quantize8): a scale for each 128 columns of a row,
    or with ``tiles`` for 128 x 128 values.  order: "rows" gives the pair (codes,
    scales) of X, "columns" that of X transposed, "both" the two pairs from one
    read of X."""
    if order not in ("rows", "columns", "both"):
        raise ValueError("order must be 'rows', 'columns' or 'both'")
    return T._run(_call().quantize_8bit, X, stream, X, bool(tiles), order != "columns", order != "rows")


def matmul_8bit(A, B, *, out_dtype=None, out=None, stream=None):
    """Y = A B^T of two matrices held in 8 bits (aires_matmul8).  A: a pair (m x k
    codes, scales for each row); B: a pair (n x k codes, scales for each row or for
    128 rows).  Y has ``out_dtype`` (bfloat16 by default) unless ``out`` is given.
    A layer's Y = X W^T takes X's rows and W in tiles, its dX takes dY's rows and W
    transposed in tiles, its dW the columns of dY and of X.  Sums are in fp32, but
    for a 16-bit Y of more than 16 rows: there each eight neighbours of k are added
    with an error of up to 8 * 2^-13 of their largest product."""
    if not (isinstance(A, tuple) and len(A) == 2 and isinstance(B, tuple) and len(B) == 2):
        raise ValueError("A and B must be pairs of codes and scales")
    return T._run(_call().matmul_8bit, A[0], stream, A, B, out_dtype, out)


@dataclass
class LogProbs:
    """What ``log_probs`` returns, one float32 value a row: logp (None without
    labels), entropy, lse; top_logp (float32) and top_index (int64), rows x
    top (None for top = 0); and lse_rest (None unless asked for)."""
    logp: Any
    entropy: Any
    lse: Any
    top_logp: Any = None
    top_index: Any = None
    lse_rest: Any = None


def log_probs(Z, labels=None, *, top: int = 0, rest: bool = False, stream=None) -> LogProbs:
    """Log probabilities of the rows of scores Z (aires_log_probs): that of each
    row's label (int32 or int64; 0 for a label outside the classes), the entropy,
    and the ``top`` most probable classes, highest first, equal scores by their
    index.  A class of score -infinity is ruled out.  With ``rest``, lse_rest is
    what the rounding of lse to float32 leaves, for ``log_probs_backward``."""
    return LogProbs(*T._run(_call().log_probs, Z, stream, Z, labels, top, bool(rest)))


def log_probs_backward(Z, labels, lse, entropy=None, *, lse_rest=None, dlogp=None, dentropy=None, dz_dtype=None,
                       out=None, stream=None):
    """Gradient of the scores (aires_log_probs_backward) from those of logp and
    entropy (float32, one a row, or None), with lse and entropy as ``log_probs``
    returned them.  dZ has ``dz_dtype`` (Z's type by default) unless ``out`` is
    given, which may be Z itself.  Probabilities are exp(Z - lse - lse_rest);
    without lse_rest they are off by up to |lse| 2^-24 of themselves, which matters
    where scores lie far from zero."""
    return T._run(_call().log_probs_backward, Z, stream, Z, labels, lse, lse_rest, entropy, dlogp, dentropy, dz_dtype, out)


def grad_norm(grads, *, max_norm: float = float("inf"), stream=None):
    """Norm over a list of gradients (aires_grad_norm), contiguous float32,
    bfloat16 or float16.  Returns (norm, scale), float32 scalars on the device:
    scale = max_norm / norm where norm is larger, else 1.  ``adamw`` takes it as
    its ``grad_scale``, which spares a pass over the gradients.  An infinite
    gradient gives scale = 0 and a NaN gives NaN: ``adamw`` then takes no gradient,
    or leaves its step out."""
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    return T._run(_call().grad_norm, grads[0], stream, grads, float(max_norm))


def clip_grads(grads, max_norm: float, *, out=None, stream=None):
    """Gradients multiplied with ``grad_norm``'s scale (aires_clip_grads), in place
    or into the tensors of ``out`` (of the same shapes, any type).  Returns the norm
    before, a float32 scalar on the device."""
    grads = list(grads)
    if not grads:
        raise ValueError("no gradients")
    return T._run(_call().clip_grads, grads[0], stream, grads, grads if out is None else list(out), float(max_norm))
