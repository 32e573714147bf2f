"""Sizes chosen so that every kernel of the training calls runs, each against
64 bits, in a workspace of exactly the stated size that held NaNs (GPU)."""
import ctypes
import math
import os
import random
import re

import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from paper_2507_02006_amd import _binding as B_  # noqa: E402
from test_gpu_train import norm_data, xent_check, xent_data, xent_ref  # noqa: E402
from test_kernel_resources import code_objects, kernels  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
CODE = {F32: B_.DTYPE_F32, BF16: B_.DTYPE_BF16, F16: B_.DTYPE_F16}

WIDTHS = [50, 100, 200, 500, 1000]
# the table kept: tiles of 16 classes by the columns a wavefront holds
CLASSES = [(700, d, v) for v in (9, 30, 41, 60) for d in WIDTHS if d < 1000 or v <= 32] + [(5003, 33, 9)]
# the rows kept: fp32, and columns that are no multiple of 8
ROWS = [(t, d + 1, 2003) for t in (9, 30, 41, 60) for d in WIDTHS if d < 1000 or t <= 32]
# tiles of 32, 128 and 256 rows of scores, of 128 and 256 of the gradients; one piece of the table and several; an odd
# number of tiles of 32
TILES = [(40, 64, 600), (20, 64, 3000), (90, 72, 700), (70, 64, 601), (100, 200, 60013), (260, 130, 40009), (1001, 201, 30011), (2300, 150, 40009),
         (5001, 131, 40009), (3000, 72, 300), (9001, 40, 301), (3000, 40, 150001)]
XENT = CLASSES + ROWS + TILES

# lanes a row and columns a lane; rows that the caches keep and rows that they do not
NORM = [(3, n) for n in (30, 60, 100, 250, 500, 1000, 2000, 7000, 15000, 30000, 33000)] + \
       [(600011, 30), (300007, 60), (180001, 100), (70003, 250), (36007, 500), (18013, 1000), (9001, 2000), (2609, 7000),
        (1201, 15000), (601, 30000), (599, 33000)]


def view(x):
    return B_.Dense(x.shape[0], x.shape[1], x.stride(0), CODE[x.dtype], 0, x.data_ptr())


def xent_in(H, W, y, grads):
    """aires_linear_xent in a workspace of the size that it asks for, every byte
    of it and of the results 0xFF before (NaN in all types)."""
    lib, need = B_.load(), ctypes.c_int64()
    t, d, v = *H.shape, W.shape[0]
    B_.check(lib.aires_linear_xent_workspace(t, d, v, CODE[H.dtype], int(grads), ctypes.byref(need)), "workspace")
    work = torch.full((need.value + 4096,), 255, dtype=torch.uint8, device="cuda")
    loss, rows = torch.full((1,), math.nan, device="cuda"), torch.full((t,), math.nan, device="cuda")
    dH, dW = (torch.full_like(x, math.nan) for x in (H, W))
    h, w, dh, dw = view(H), view(W), view(dH), view(dW)
    B_.check(lib.aires_linear_xent(ctypes.byref(h), ctypes.byref(w), y.data_ptr(), 1, B_.REDUCE_MEAN, 1.0, loss.data_ptr(),
                                   rows.data_ptr(), ctypes.byref(dh) if grads else None, ctypes.byref(dw) if grads else None,
                                   work.data_ptr(), need.value, torch.cuda.current_stream().cuda_stream), "aires_linear_xent")
    assert bool((work[need.value:] == 255).all()), "written past the workspace"
    return loss[0], rows, dH, dW


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("t,d,v", XENT)
def test_linear_xent(t, d, v, dt):
    H, W, y = xent_data(t, d, v, dt, 3 * t + d + 11 * v)
    y[0], y[-1] = v - 1, 0
    ref = xent_ref(H, W, y)
    H, W, y = H.cuda(), W.cuda(), y.cuda()
    for grads in (True, False):
        got = aires.linear_xent(H, W, y, grads=grads)
        xent_check(got, ref, grads)
        for a, b in zip((got.loss, got.row_loss, got.dH, got.dW), xent_in(H, W, y, grads)):
            assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("seed", range(24))
def test_linear_xent_sizes_at_random(seed):
    """Sizes next to what fills tiles, steps and pieces, and any others."""
    rng = random.Random(seed)

    def size(lo, hi):
        x = round(math.exp(rng.uniform(math.log(lo), math.log(hi))))
        to = rng.choice([1, 8, 16, 32, 64, 256])
        return max(lo, min(hi, (x + to - 1) // to * to + (rng.choice([-1, 0, 0, 1]) if to > 1 else 0)))

    for _ in range(8):
        dt, d, v = rng.choice([F32, BF16, F16]), size(1, 1100), size(2, 30000)
        t = size(1, max(2, min(6000, 12000000 // v)))
        H, W, y = xent_data(t, d, v, dt, seed)
        y[rng.randrange(t)] = rng.randrange(v)
        print(seed, t, d, v, dt, flush=True)
        xent_check(aires.linear_xent(H.cuda(), W.cuda(), y.cuda()), xent_ref(H, W, y))


@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("t,d,v", [(700, 100, 41), (70, 500, 60), (20, 131, 3000), (60, 200, 2000), (40, 64, 600),
                                   (100, 200, 60013), (1001, 200, 30011)])
def test_linear_xent_of_rows_that_are_no_numbers_and_have_no_label(t, d, v, dt):
    """They change no loss and no other row's gradient, and their own are 0."""
    H, W, y = xent_data(t, d, v, dt, t + v)
    off = torch.zeros(t, dtype=torch.bool)
    off[[0, 2, t // 2, t - 1]] = True
    y[off] = torch.tensor([-1, v, -100, 2 ** 40])
    y[1] = 1
    H, W, y = H.cuda(), W.cuda(), y.cuda()
    bad = H.clone()
    bad[0], bad[2, d // 2], bad[t // 2, 0], bad[t - 1] = math.nan, math.inf, -math.inf, math.nan
    for grads in (True, False):
        clean, got = (aires.linear_xent(x, W, y, grads=grads) for x in (H, bad))
        assert torch.equal(got.loss, clean.loss) and torch.equal(got.row_loss, clean.row_loss)
        assert not got.row_loss[off.cuda()].any()
        if grads:
            assert torch.equal(got.dH, clean.dH) and not got.dH[off.cuda()].any()


@pytest.mark.parametrize("t,d,v", [(70, 9, 9000013), (300, 9, 9000013)])
def test_linear_xent_table_packed_in_pieces(t, d, v):
    """Columns that have to be copied and a copy of more than 1 GiB: the same
    bits as where the table is read as it lies, in as many columns as a step has."""
    g = torch.Generator(device="cuda").manual_seed(t)
    for dt in (BF16, F16):
        wide = [torch.zeros(n, 64, dtype=dt, device="cuda") for n in (t, v)]
        for x in wide:
            x[:, :d] = torch.randn(x.shape[0], d, generator=g, device="cuda")
        H, W = (x[:, :d].contiguous() for x in wide)
        y = torch.randint(-1, v, (t,), generator=g, device="cuda")
        for grads in (True, False):
            a, b = aires.linear_xent(H, W, y, grads=grads), aires.linear_xent(*wide, y, grads=grads)
            assert torch.equal(a.loss, b.loss) and torch.equal(a.row_loss, b.row_loss)
            assert bool(a.row_loss[y >= 0].isfinite().all()) and bool((a.row_loss[y >= 0] > 0).all())
            if grads:
                assert torch.equal(a.dH, b.dH[:, :d]) and torch.equal(a.dW, b.dW[:, :d])


def test_linear_xent_planes_of_a_table_made_in_pieces():
    t, d, v = 70, 8, 12000007  # (planes of 1.2e9 bytes)
    g = torch.Generator(device="cuda").manual_seed(1)
    H, W = torch.randn(t, d, generator=g, device="cuda"), torch.randn(v, d, generator=g, device="cuda")
    y = torch.randint(0, v, (t,), generator=g, device="cuda")
    y[0], y[1], y[2] = 0, v - 1, -1
    got = aires.linear_xent(H, W, y)
    alone = aires.linear_xent(H, W, y, grads=False)
    assert torch.equal(alone.row_loss, got.row_loss)
    h, there = H.double(), (y >= 0).double()
    lse = torch.full((t,), -math.inf, dtype=torch.float64, device="cuda")
    step = 1 << 20
    for v0 in range(0, v, step):
        lse = torch.logaddexp(lse, torch.logsumexp(h @ W[v0:v0 + step].double().t(), 1))
    target = (h * W[y.clamp(min=0)].double()).sum(1)
    ez = (d + 8) * U * (h.abs() @ W.abs().amax(0).double())
    el = ez + 256 * U * (1 + lse.abs() + 40)  # (no score is above 40)
    assert bool(((got.row_loss.double() - (lse - target) * there).abs() <= 2 * el * there).all())
    c = there.sum()
    dH, eH = torch.zeros(t, d, dtype=torch.float64, device="cuda"), torch.zeros(t, d, dtype=torch.float64, device="cuda")
    for v0 in range(0, v, step):
        w = W[v0:v0 + step].double()
        z = h @ w.t()
        assert float(z.abs().max()) < 40
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p)
        here = ((y >= v0) & (y < v0 + w.shape[0])).nonzero().squeeze(1)
        hot[here, y[here] - v0] = 1
        dz = (p - hot) * there[:, None] / c
        # as for any size: a score off by ez, lse by el; dz kept in planes; chains of 1024 additions
        e = (p * (2 * (ez + el)[:, None] + 16 * U) + U * (p - hot).abs() + 2.0 ** -40 + 2 * U * hot) * there[:, None] / c
        dH += dz @ w
        eH += e @ w.abs() + 1024 * U * (dz.abs() @ w.abs())
        dW, eW = dz.t() @ h, e.t() @ h.abs() + 1024 * U * (dz.abs().t() @ h.abs())
        assert bool(((got.dW[v0:v0 + step].double() - dW).abs() <= eW + U * dW.abs()).all()), v0
    assert bool(((got.dH.double() - dH).abs() <= eH + U * dH.abs()).all())


@pytest.mark.parametrize("m,n", NORM)
def test_layer_norm(m, n):
    """Rows of a large matrix as on their own (those are held against 64 bits
    elsewhere), and the weights' gradients against 64 bits."""
    x, gamma, beta = norm_data(m, n, F16, m + n)
    dy = torch.randn(m, n, generator=torch.Generator().manual_seed(n)).to(F16)
    X, D, gamma, beta = x.cuda(), dy.cuda(), gamma.cuda(), beta.cuda()
    Y, mean, rstd = aires.layer_norm(X, gamma, beta)
    dX, dgamma, dbeta = aires.layer_norm_backward(D, X, mean, rstd, gamma)
    for at in (0, m // 2, m - 1):
        some = slice(at, at + 1)
        one = aires.layer_norm(X[some], gamma, beta)
        assert all(torch.equal(a[some], b) for a, b in zip((Y, mean, rstd), one))
        assert torch.equal(dX[some], aires.layer_norm_backward(D[some], X[some], mean[some], rstd[some], gamma)[0])
    step = max(1, (1 << 26) // n)
    total, size, sums, sizes = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(4))
    for r in range(0, m, step):
        d, mu, r_ = D[r:r + step].double(), mean[r:r + step].double()[:, None], rstd[r:r + step].double()[:, None]
        xh = (X[r:r + step].double() - mu) * r_
        total += (d * xh).sum(0)
        size += (d * xh).abs().sum(0) + (d.abs() * (X[r:r + step].double().abs() + mu.abs()) * r_).sum(0) / 64
        sums += d.sum(0)
        sizes += d.abs().sum(0)
    # chains of at most 512 additions; xh is off by 4 U of its terms, 1/64 of 256 U
    assert bool(((dgamma.double() - total).abs() <= 512 * U * size).all())
    assert bool(((dbeta.double() - sums).abs() <= 512 * U * sizes).all())
    # in a workspace of exactly the stated size that held NaNs
    lib, need = B_.load(), ctypes.c_int64()
    B_.check(lib.aires_layer_norm_workspace(m, n, ctypes.byref(need)), "workspace")
    work = torch.full((need.value + 4096,), 255, dtype=torch.uint8, device="cuda")
    out, dg, db = torch.full_like(X, math.nan), torch.full_like(gamma, math.nan), torch.full_like(gamma, math.nan)
    a, b, c = view(D), view(X), view(out)
    B_.check(lib.aires_layer_norm_backward(ctypes.byref(a), ctypes.byref(b), mean.data_ptr(), rstd.data_ptr(), gamma.data_ptr(), 0,
                                           ctypes.byref(c), dg.data_ptr(), db.data_ptr(), work.data_ptr(), need.value,
                                           torch.cuda.current_stream().cuda_stream), "aires_layer_norm_backward")
    assert bool((work[need.value:] == 255).all()), "written past the workspace"
    assert torch.equal(out, dX) and torch.equal(dg, dgamma) and torch.equal(db, dbeta)


OURS = re.compile(r"^k_(ln_|adamw_|few$|count$|scores$|rows$|total$|gradients$|finish$|zero$|pack$)")


def built():
    """(name, template arguments) of the training calls' kernels in the library."""
    with open(os.path.join(os.path.dirname(B_.__file__), "libaires.so"), "rb") as f:
        names = {n for elf in code_objects(f.read()) for n in kernels(elf)}
    found = set()
    for n in names:
        m = re.search(r"_GLOBAL__N_1(\d+)(k_\w*)", n)
        if m:
            name, rest = m[2][:int(m[1])], m[2][int(m[1]):]
            args = re.match(r"I((?:L[a-z]\d+E)+)E", rest)
            if OURS.match(name):
                found.add((name, tuple(int(x) for x in re.findall(r"L[a-z](\d+)E", args[1])) if args else ()))
    return found


def test_every_kernel_runs():
    """The sizes above, and the few calls that have none, launch every kernel
    that the library holds for these calls."""
    from torch.profiler import ProfilerActivity, profile
    want = built()
    assert len(want) > 200

    def calls():
        for t, d, v in XENT:
            for dt in (F32, BF16, F16):
                H, W = torch.zeros(t, d, dtype=dt, device="cuda"), torch.zeros(v, d, dtype=dt, device="cuda")
                y = torch.zeros(t, dtype=torch.int64, device="cuda")
                for grads in (True, False):
                    aires.linear_xent(H, W, y, grads=grads)
        aires.linear_xent(torch.zeros(0, 8, device="cuda"), torch.zeros(300, 8, device="cuda"), y[:0])
        for m, n in NORM:
            X = torch.zeros(m, n, dtype=F16, device="cuda")
            _, mean, rstd = aires.layer_norm(X)
            aires.layer_norm_backward(X, X, mean, rstd)
        aires.layer_norm(torch.empty(3, 0, device="cuda"))
        for bits in (8, 32):
            p = [torch.zeros(300, device="cuda")]
            aires.adamw(p, [p[0].clone()], *aires.adamw_state(p, bits=bits), step=1, lr=0.1)
        torch.cuda.synchronize()

    calls()
    with profile(activities=[ProfilerActivity.CUDA]) as trace:
        calls()
    ran = set()
    for e in trace.events():
        m = re.search(r"aires::kern::\(anonymous namespace\)::(k_\w+)(?:<([^>]*)>)?\(", e.name)
        if m and OURS.match(m[1]):
            args = [x.strip() for x in (m[2] or "").split(",") if x.strip()]
            ran.add((m[1], tuple({"true": 1, "false": 0}.get(x) if x in ("true", "false") else int(x) for x in args)))
    assert ran <= want, sorted(ran - want)
    assert ran == want, sorted(want - ran)
