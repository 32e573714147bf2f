"""Refusals of the layers' calls at the C boundary (CPU: every one of these fails
before anything is launched)."""
import ctypes
import math

import pytest

from paper_2507_02006_amd import _binding as B_

FAKE = 4096  # an aligned address that no call here may read


@pytest.fixture(scope="module")
def lib():
    return B_.load()


def dense(m, n, ld=None, dtype=0, data=FAKE):
    return B_.Dense(m, n, n if ld is None else ld, dtype, 0, data)


def held(m, n, tile=1, ld=None, lds=None, codes=FAKE, scales=FAKE):
    return B_.Dense8(m, n, n if ld is None else ld, codes, scales, -(-n // 128) if lds is None else lds, tile, 0)


def ref(x):
    return ctypes.byref(x) if x is not None else None


BAD_ROWS = [dense(2, 3, dtype=7), dense(2, 3, dtype=3), dense(2, 3, ld=2), dense(2, 3, data=None)]


def test_struct_sizes_match_the_header():
    assert ctypes.sizeof(B_.Dense8) == 56 and ctypes.sizeof(B_.GradTensor) == 32
    text = open(B_.HEADER).read()
    assert "#define AIRES_BLOCK8 %d" % B_.BLOCK8 in text and "#define AIRES_MAX_TOP %d" % B_.MAX_TOP in text


def test_rms_norm(lib):
    def call(X=dense(2, 3), R=None, S=None, Y=dense(2, 3), Y8=None, eps=1e-6, wt=0, gamma=None):
        rc = lib.aires_rms_norm(ref(X), ref(R), gamma, wt, eps, ref(S), ref(Y), ref(Y8), None, None)
        assert rc == B_.OK or lib.aires_last_error()
        return rc

    for X in [None] + BAD_ROWS:
        assert call(X=X) == B_.E_INVALID_ARG
    assert call(X=dense(-1, 3), Y=dense(-1, 3)) == B_.E_DIM
    assert call(Y=dense(2, 4)) == call(Y=None, Y8=held(2, 4)) == call(Y=None, Y8=held(3, 3)) == B_.E_DIM
    assert call(Y=None) == call(Y8=held(2, 3)) == B_.E_INVALID_ARG
    assert call(Y=None, Y8=held(2, 3, tile=128)) == call(Y=None, Y8=held(2, 3, tile=5)) == B_.E_INVALID_ARG
    assert call(Y=None, Y8=held(2, 3, ld=2)) == call(Y=None, Y8=held(2, 300, lds=2)) == B_.E_INVALID_ARG
    assert call(Y=None, Y8=held(2, 3, codes=None)) == call(Y=None, Y8=held(2, 3, scales=None)) == B_.E_INVALID_ARG
    assert call(Y=None, Y8=held(2, 3, scales=FAKE + 2)) == B_.E_INVALID_ARG
    assert call(R=dense(2, 3)) == call(S=dense(2, 3)) == B_.E_INVALID_ARG
    assert call(R=dense(2, 4), S=dense(2, 3)) == call(R=dense(2, 3), S=dense(3, 3)) == B_.E_DIM
    # the sum in the place of an input, in another type or with another stride
    assert call(R=dense(2, 3), S=dense(2, 3, dtype=1)) == call(R=dense(2, 3, data=8192), S=dense(2, 3, ld=4)) == B_.E_INVALID_ARG
    assert call(eps=-1.0) == call(eps=math.nan) == call(eps=math.inf) == call(wt=3) == B_.E_INVALID_ARG
    big = dense(1, 2 ** 30 + 1)
    assert call(X=big, Y=big) == call(X=dense(2 ** 40 + 1, 1), Y=dense(2 ** 40 + 1, 1)) == B_.E_UNSUPPORTED
    none = dense(0, 3, data=None)
    assert call(X=none, Y=none) == call(X=none, Y=None, Y8=held(0, 3, codes=None, scales=None)) == B_.OK


def test_rms_norm_backward(lib):
    need = ctypes.c_int64()
    assert lib.aires_rms_norm_workspace(50, 7, ctypes.byref(need)) == B_.OK and need.value > 0
    S = dense(50, 7)

    def call(dY=S, S=S, rstd=FAKE, dS=None, dX=dense(50, 7, data=8192), dg=FAKE, ws=FAKE, n=need.value, wt=0):
        return lib.aires_rms_norm_backward(ref(dY), ref(S), rstd, FAKE, wt, ref(dS), ref(dX), dg, ws, n, None)

    assert call(dY=None) == call(S=None) == call(rstd=None) == call(wt=3) == B_.E_INVALID_ARG
    assert call(dY=dense(50, 8)) == call(dX=dense(49, 7)) == call(dS=dense(50, 6)) == B_.E_DIM
    assert call(dS=dense(50, 7, data=8192, dtype=1)) == call(dS=dense(50, 7, data=8192, ld=9)) == B_.E_INVALID_ARG
    assert call(ws=None) == call(ws=FAKE + 4) == B_.E_INVALID_ARG
    assert call(n=need.value - 1) == B_.E_CAPACITY
    assert lib.aires_rms_norm_workspace(-1, 7, ctypes.byref(need)) == B_.E_DIM
    assert lib.aires_rms_norm_workspace(1, 7, None) == B_.E_INVALID_ARG
    assert lib.aires_rms_norm_workspace(1, 2 ** 30 + 1, ctypes.byref(need)) == B_.E_UNSUPPORTED


def test_quantize(lib):
    call = lambda X=dense(5, 300), Q=held(5, 300), Qt=None: lib.aires_quantize8(ref(X), ref(Q), ref(Qt), None)  # noqa: E731
    assert call(X=None) == call(Q=None) == call(X=dense(5, 300, ld=299)) == call(X=dense(5, 300, dtype=3)) == B_.E_INVALID_ARG
    assert call(Q=held(5, 299)) == call(Q=held(300, 5)) == call(Q=None, Qt=held(5, 300)) == B_.E_DIM
    assert call(Qt=held(300, 5, tile=128)) == call(Q=held(5, 300, tile=2)) == call(Q=held(5, 300, lds=2)) == B_.E_INVALID_ARG
    wide = dense(1, 2 ** 30 + 1)
    assert call(X=wide, Q=held(1, 2 ** 30 + 1)) == B_.E_UNSUPPORTED


@pytest.mark.parametrize("m,n,k", [(5, 7, 300), (100, 80, 4096), (300, 300, 4097), (4000, 3000, 512)])
def test_matmul(lib, m, n, k):
    need = ctypes.c_int64()
    A, B, Y = held(m, k), held(n, k, tile=128), dense(m, n)
    size = lambda A=A, B=B, dtype=0: lib.aires_matmul8_workspace(ref(A), ref(B), dtype, ctypes.byref(need))  # noqa: E731
    assert size() == B_.OK
    bytes_ = need.value
    assert (bytes_ > 0) == (m > 16 and (k % 16 != 0 or (m, n) == (100, 80)))

    def call(A=A, B=B, Y=Y, ws=FAKE, n=bytes_):
        return lib.aires_matmul8(ref(A), ref(B), ref(Y), ws, n, None)

    for bad in (None, held(m, k, tile=128), held(m, k, tile=3), held(m, k, ld=k - 1), held(m, k, codes=None), held(m, k, lds=0)):
        assert call(A=bad) == size(A=bad) == B_.E_INVALID_ARG
    assert call(B=None) == call(Y=None) == call(Y=dense(m, n, dtype=5)) == size(dtype=3) == B_.E_INVALID_ARG
    assert call(B=held(n, k + 1)) == size(B=held(n, k + 1)) == call(Y=dense(m, n + 1)) == call(Y=dense(m + 1, n)) == B_.E_DIM
    assert call(A=held(m, k, ld=2 ** 23 + 1)) == call(B=held(n, k, lds=2 ** 21 + 1)) == B_.E_UNSUPPORTED
    if bytes_:
        assert call(ws=None) == call(ws=FAKE + 8) == B_.E_INVALID_ARG
        assert call(n=bytes_ - 1) == B_.E_CAPACITY
    assert lib.aires_matmul8_workspace(ref(A), ref(B), 0, None) == B_.E_INVALID_ARG


def test_matmul_sizes(lib):
    need = ctypes.c_int64()
    q = lambda m, n, k, t=1: lib.aires_matmul8_workspace(ref(held(m, k)), ref(held(n, k)), t, ctypes.byref(need))  # noqa: E731
    assert q(8, 2 ** 26, 64) == q(2 ** 26, 8, 64) == q(2, 2, 2 ** 23) == B_.OK
    assert q(8, 2 ** 26 + 1, 64) == q(2 ** 26 + 1, 8, 64) == q(2, 2, 2 ** 23 + 1) == q(2 ** 20, 2 ** 17, 64) == B_.E_UNSUPPORTED
    assert q(0, 5, 64) == q(5, 0, 64) == q(5, 5, 0) == B_.OK and need.value == 0
    # partial sums stay within 64 MB, copies within the operands' size
    for m, n, k in ((1000, 520, 65536), (17, 17, 2 ** 23), (2000, 2000, 100000), (4096, 8192, 4096)):
        for t in (0, 1):
            assert q(m, n, k, t) == B_.OK and need.value <= (64 << 20) + (m + n) * (k + 16), (m, n, k)


def test_log_probs(lib):
    need = ctypes.c_int64()
    size = lambda t, v, top: lib.aires_log_probs_workspace(t, v, top, ctypes.byref(need))  # noqa: E731
    assert size(3, 262144, 10) == B_.OK and need.value > 0
    n = need.value
    Z = dense(3, 262144)

    def call(Z=Z, labels=FAKE, top=10, logp=FAKE, tl=FAKE, ti=FAKE, ws=FAKE, n=n):
        return lib.aires_log_probs(ref(Z), labels, 0, top, logp, FAKE, FAKE, tl, ti, ws, n, None)

    assert call(Z=None) == call(Z=dense(3, 262144, dtype=9)) == call(Z=dense(3, 262144, ld=7)) == B_.E_INVALID_ARG
    assert call(labels=None) == call(logp=None) == call(tl=None) == call(ti=None) == B_.E_INVALID_ARG
    assert call(top=-1) == call(top=65) == B_.E_INVALID_ARG
    assert call(Z=dense(3, 5)) == call(Z=dense(3, 0)) == B_.E_DIM
    assert call(ws=None) == call(ws=FAKE + 4) == B_.E_INVALID_ARG
    assert call(n=n - 1) == B_.E_CAPACITY
    assert size(1, 2 ** 30, 0) == size(2 ** 40 + 1, 8, 0) == B_.E_UNSUPPORTED
    assert size(-1, 8, 0) == size(3, 0, 0) == size(3, 4, 5) == B_.E_DIM
    assert size(3, 8, 65) == B_.E_INVALID_ARG and size(0, 0, 5) == B_.OK
    assert lib.aires_log_probs_workspace(1, 1, 1, None) == B_.E_INVALID_ARG


def test_log_probs_backward(lib):
    def call(Z=dense(3, 50), labels=FAKE, lse=FAKE, h=FAKE, da=FAKE, db=FAKE, dZ=dense(3, 50, data=8192)):
        return lib.aires_log_probs_backward(ref(Z), labels, 0, lse, h, da, db, ref(dZ), None)

    assert call(Z=None) == call(dZ=None) == call(lse=None) == call(h=None) == call(labels=None) == B_.E_INVALID_ARG
    assert call(dZ=dense(3, 51)) == call(dZ=dense(4, 50)) == call(Z=dense(3, 0), dZ=dense(3, 0)) == B_.E_DIM
    assert call(dZ=dense(3, 50, dtype=1)) == call(dZ=dense(3, 50, ld=51)) == B_.E_INVALID_ARG  # in Z's place, another type or stride


def test_grad_norm(lib):
    need = ctypes.c_int64()
    assert lib.aires_grad_norm_workspace(3, ctypes.byref(need)) == B_.OK and need.value > 0
    n = need.value

    def call(rows=None, count=None, most=1.0, norm=FAKE, ws=FAKE, n=n, clip=False):
        rows = rows if rows is not None else [(4, FAKE, FAKE, 0, 0)]
        table = (B_.GradTensor * max(1, len(rows)))(*[B_.GradTensor(*r) for r in rows])
        count = len(rows) if count is None else count
        if clip:
            return lib.aires_clip_grads(table, count, most, norm, ws, n, None)
        return lib.aires_grad_norm(table, count, most, norm, None, ws, n, None)

    for clip in (False, True):
        assert call(most=-1.0, clip=clip) == call(most=math.nan, clip=clip) == call(norm=None, clip=clip) == B_.E_INVALID_ARG
        assert call(rows=[(4, None, FAKE, 0, 0)], clip=clip) == call(rows=[(4, FAKE, FAKE, 5, 0)], clip=clip) == B_.E_INVALID_ARG
        assert call(rows=[(-4, FAKE, FAKE, 0, 0)], clip=clip) == B_.E_DIM
        assert call(rows=[(2 ** 35 + 1, FAKE, FAKE, 0, 0)], clip=clip) == call(count=2 ** 24 + 1, clip=clip) == B_.E_UNSUPPORTED
        assert call(count=-1, clip=clip) == call(ws=None, clip=clip) == call(ws=FAKE + 8, clip=clip) == B_.E_INVALID_ARG
        assert call(n=100, clip=clip) == B_.E_CAPACITY
    assert lib.aires_grad_norm(None, 1, 1.0, FAKE, None, FAKE, n, None) == B_.E_INVALID_ARG
    assert call(rows=[(4, FAKE, None, 0, 0)], clip=True) == call(rows=[(4, FAKE, FAKE, 0, 3)], clip=True) == B_.E_INVALID_ARG
    assert call(rows=[(4, FAKE, FAKE, 0, 1)], clip=True) == B_.E_INVALID_ARG          # in place, another type
    # outs that overlap each other, a gradient of another tensor, or their own not exactly
    for rows in ([(4, FAKE, FAKE, 0, 0), (4, FAKE, FAKE, 0, 0)], [(4, FAKE, 8192, 0, 0), (4, 9000, 8200, 0, 0)],
                 [(8, FAKE, 8192, 0, 0), (8, 8192 + 28, 16384, 0, 0)], [(8, FAKE, FAKE + 4, 0, 0)], [(8, FAKE, FAKE - 4, 0, 0)],
                 [(8, FAKE, 8192, 0, 0), (64, 8000, 16384, 0, 0)]):
        assert call(rows=rows, clip=True) == B_.E_INVALID_ARG, rows
    assert lib.aires_grad_norm_workspace(-1, ctypes.byref(need)) == lib.aires_grad_norm_workspace(1, None) == B_.E_INVALID_ARG


def test_adamw_scaled(lib):
    assert lib.aires_adamw_scaled(None, 1, None, None, None) == B_.E_INVALID_ARG
    opts = B_.AdamWOpts(ctypes.sizeof(B_.AdamWOpts), 0, 1, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1.0)
    assert lib.aires_adamw_scaled(None, 0, ctypes.byref(opts), FAKE, None) == B_.OK
