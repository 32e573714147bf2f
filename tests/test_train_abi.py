"""Refusals of the training calls at the C boundary (CPU: every one of these
fails before anything is launched)."""
import ctypes

import pytest

from paper_2507_02006_amd import _binding as B_

FAKE = 4096  # an aligned address that no call here may read


@pytest.fixture(scope="module")
def lib():
    return B_.load()


def dense(m, n, ld=None, dtype=0, data=FAKE):
    return B_.Dense(m, n, n if ld is None else ld, dtype, 0, data)


def ref(x):
    return ctypes.byref(x) if x is not None else None


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(B_.Dense) == 40
    assert ctypes.sizeof(B_.AdamWTensor) == 80
    assert ctypes.sizeof(B_.AdamWOpts) == 64


@pytest.mark.parametrize("X,Y,eps,mean,rstd,want", [
    (None, dense(2, 3), 1e-5, None, None, B_.E_INVALID_ARG),
    (dense(2, 3), None, 1e-5, None, None, B_.E_INVALID_ARG),
    (dense(2, 3, dtype=7), dense(2, 3), 1e-5, None, None, B_.E_INVALID_ARG),
    (dense(2, 3, ld=2), dense(2, 3), 1e-5, None, None, B_.E_INVALID_ARG),
    (dense(2, 3, data=None), dense(2, 3), 1e-5, None, None, B_.E_INVALID_ARG),
    (dense(-1, 3), dense(-1, 3), 1e-5, None, None, B_.E_DIM),
    (dense(2, 3), dense(2, 4), 1e-5, None, None, B_.E_DIM),
    (dense(1, 2 ** 31), dense(1, 2 ** 31), 1e-5, None, None, B_.E_UNSUPPORTED),
    (dense(2, 3), dense(2, 3), -1.0, None, None, B_.E_INVALID_ARG),
    (dense(2, 3), dense(2, 3), float("nan"), None, None, B_.E_INVALID_ARG),
    (dense(2, 3), dense(2, 3), 1e-5, FAKE, None, B_.E_INVALID_ARG),
])
def test_layer_norm(lib, X, Y, eps, mean, rstd, want):
    assert lib.aires_layer_norm(ref(X), None, None, 0, eps, ref(Y), mean, rstd, None) == want
    assert lib.aires_last_error()


def test_layer_norm_backward(lib):
    X, need = dense(50, 7), ctypes.c_int64()
    assert lib.aires_layer_norm_workspace(50, 7, ctypes.byref(need)) == B_.OK and need.value > 0
    call = lambda dY=X, mean=FAKE, dX=X, dg=FAKE, ws=FAKE, n=need.value, wt=0: lib.aires_layer_norm_backward(  # noqa: E731
        ref(dY), ref(X), mean, FAKE, FAKE, wt, ref(dX), dg, None, ws, n, None)
    assert call(dY=dense(50, 8)) == B_.E_DIM
    assert call(dX=dense(49, 7)) == B_.E_DIM
    assert call(mean=None) == B_.E_INVALID_ARG
    assert call(wt=3) == B_.E_INVALID_ARG
    assert call(ws=None) == B_.E_INVALID_ARG
    assert call(ws=FAKE + 4) == B_.E_INVALID_ARG
    assert call(n=need.value - 1) == B_.E_CAPACITY
    assert lib.aires_layer_norm_workspace(-1, 7, ctypes.byref(need)) == B_.E_DIM
    assert lib.aires_layer_norm_workspace(1, 7, None) == B_.E_INVALID_ARG


@pytest.mark.parametrize("t,d,v,dtype", [(5, 8, 9, 0), (100, 64, 3000, 1), (300, 40, 7, 2), (9, 1000, 4000, 0),
                                         (700, 130, 700, 0), (1, 1, 1, 1)])
def test_linear_xent(lib, t, d, v, dtype):
    H, W = dense(t, d, dtype=dtype), dense(v, d, dtype=dtype)
    need = ctypes.c_int64()
    assert lib.aires_linear_xent_workspace(t, d, v, dtype, 1, ctypes.byref(need)) == B_.OK and need.value > 0
    n = need.value
    assert lib.aires_linear_xent_workspace(t, d, v, dtype, 0, ctypes.byref(need)) == B_.OK and need.value <= n

    def call(H=H, W=W, labels=FAKE, red=0, scale=1.0, loss=FAKE, dH=H, dW=W, ws=FAKE, n=n):
        return lib.aires_linear_xent(ref(H), ref(W), labels, 0, red, scale, loss, None, ref(dH), ref(dW), ws, n, None)

    assert call(H=None) == B_.E_INVALID_ARG
    assert call(W=dense(v, d + 1, dtype=dtype)) == B_.E_DIM
    assert call(W=dense(v, d, dtype=(dtype + 1) % 3)) == B_.E_DIM
    assert call(W=dense(0, d, dtype=dtype)) == B_.E_DIM
    assert call(dW=None) == B_.E_INVALID_ARG
    assert call(dH=dense(t + 1, d, dtype=dtype)) == B_.E_DIM
    assert call(dH=dense(t, d, dtype=(dtype + 1) % 3)) == B_.E_DIM
    assert call(labels=None) == B_.E_INVALID_ARG
    assert call(loss=None) == B_.E_INVALID_ARG
    assert call(red=2) == B_.E_INVALID_ARG
    assert call(scale=float("inf")) == B_.E_INVALID_ARG
    assert call(ws=None) == B_.E_INVALID_ARG
    assert call(n=n - 1) == B_.E_CAPACITY


def test_linear_xent_sizes(lib):
    n = ctypes.c_int64()
    q = lambda t, d, v: lib.aires_linear_xent_workspace(t, d, v, 1, 1, ctypes.byref(n))  # noqa: E731
    assert q(2 ** 31, 8, 8) == q(8, 8, 2 ** 31) == q(8, 2 ** 21, 8) == B_.E_UNSUPPORTED
    assert q(2 ** 30, 64, 2 ** 30) == B_.E_UNSUPPORTED  # more tiles than a launch holds
    assert q(-1, 8, 8) == q(8, 0, 8) == q(8, 8, 0) == B_.E_DIM
    assert q(0, 8, 0) == B_.OK
    assert lib.aires_linear_xent_workspace(8, 8, 8, 5, 1, ctypes.byref(n)) == B_.E_INVALID_ARG


def test_linear_xent_sizes_that_no_launch_holds(lib):
    n = ctypes.c_int64()
    q = lambda t, d, v, g=1: lib.aires_linear_xent_workspace(t, d, v, 1, g, ctypes.byref(n))  # noqa: E731
    assert q(2 ** 29 + 1, 8, 100) == q(2 ** 20, 2 ** 20, 8) == q(8, 2 ** 20, 2 ** 20) == B_.E_UNSUPPORTED
    assert q(2 ** 29, 8, 100) == q(2 ** 19, 8, 2 ** 30, 0) == B_.OK


def test_adamw(lib):
    o = dict(struct_size=ctypes.sizeof(B_.AdamWOpts), seed=0, step=1, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
             weight_decay=0.0, grad_scale=1.0)

    def call(t=None, count=1, **kw):
        row = B_.AdamWTensor(4, FAKE, FAKE, FAKE, FAKE, None, None, None, 0, 0, 0, 0)
        for k, x in (t or {}).items():
            setattr(row, k, x)
        opts = B_.AdamWOpts(*({**o, **kw}[f] for f, _ in B_.AdamWOpts._fields_))
        return lib.aires_adamw(ctypes.addressof(row), count, ctypes.byref(opts), None)

    assert call(count=0) == B_.OK
    assert call(t=dict(n=0)) == B_.OK
    assert lib.aires_adamw(None, 1, None, None) == B_.E_INVALID_ARG
    assert call(struct_size=8) == call(count=-1) == call(step=0) == B_.E_INVALID_ARG
    for bad in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=float("nan")), dict(grad_scale=float("inf")),
                dict(weight_decay=float("nan")), dict(beta1=float("nan"))):
        assert call(**bad) == B_.E_INVALID_ARG
    for bad in (dict(param=None), dict(grad=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(param_dtype=9),
                dict(grad_dtype=-1), dict(exp_avg_scale=FAKE), dict(copy=FAKE, copy_dtype=4)):
        assert call(t=bad) == B_.E_INVALID_ARG
    assert call(t=dict(n=-1)) == B_.E_DIM
    assert call(t=dict(n=2 ** 41)) == B_.E_UNSUPPORTED


def test_layer_norm_sizes(lib):
    n = ctypes.c_int64()
    q = lambda m, c: lib.aires_layer_norm_workspace(m, c, ctypes.byref(n))  # noqa: E731
    assert q(1, 2 ** 30) == q(2 ** 40, 1) == B_.OK
    assert q(1, 2 ** 30 + 1) == q(1, 2 ** 31 - 1) == q(2 ** 40 + 1, 1) == q(2 ** 62, 2 ** 31) == B_.E_UNSUPPORTED


def test_adamw_sizes(lib):
    row = B_.AdamWTensor(2 ** 35 + 1, FAKE, FAKE, FAKE, FAKE, None, None, None, 0, 0, 0, 0)
    opts = B_.AdamWOpts(ctypes.sizeof(B_.AdamWOpts), 0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0)
    assert lib.aires_adamw(ctypes.addressof(row), 1, ctypes.byref(opts), None) == B_.E_UNSUPPORTED
