"""The layers' calls where their arguments end (GPU): no rows, factors and scales that are
not ordinary numbers, scores far from zero."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from test_gpu_layers import BF16, F16, F32, F8, U, equal, logp_ref, logp_tolerance, near, rand, rounded  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v", [5, 300, 2049, 100000])
def test_log_probs_of_no_rows(v):
    z, labels = torch.empty(0, v, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    for top in (0, 1, 5):
        r = aires.log_probs(z, labels, top=top)
        assert r.logp.shape == r.entropy.shape == r.lse.shape == (0,)
        assert top == 0 or r.top_index.shape == r.top_logp.shape == (0, top)
    assert aires.log_probs_backward(z, labels, r.lse, r.entropy, dlogp=r.logp, dentropy=r.entropy).shape == (0, v)


@pytest.mark.parametrize("n", [40, 1500, 20000])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_norm_of_squares_past_the_range(n, kind):
    """Finite values whose squares' sum is none: q = 0 and zeros, in that row alone."""
    x = rand((5, n), n, kind)
    want, _, p = aires.rms_norm(x.cuda())
    x[1], x[3] = 3e19, 1e17                  # (20000 times 1e34 is in fp32's range)
    for out in (kind, F8):
        y, _, q = aires.rms_norm(x.cuda(), out_dtype=out)
        y = y[0].float() if out == F8 else y
        assert float(q[1]) == 0 and not bool(y[1].any()) and abs(float(q[3]) * float(x[3, 0]) - 1) < 400 * U
        assert bool((q[::2] == p[::2]).all())
    y = aires.rms_norm(x.cuda())[0]
    assert bool((y[::2] == want[::2]).all())


# ------------------------------------------------- AdamW's factor of the gradients

def step(bits, steps=2, grads=None, copies=False, start=0, **kw):
    """Steps over tensors with a whole and a partial span: parameters, moments and copies."""
    shapes = [(33, 170), (300,), (4096,)]
    params = [rand(s, 1 + i).cuda().to(t) for i, (s, t) in enumerate(zip(shapes, (F32, BF16, F32)))]
    if grads is None:
        grads = [rand(s, 5 + i, t).cuda() for i, (s, t) in enumerate(zip(shapes, (BF16, F16, F32)))]
    m, v = aires.adamw_state(params, bits=bits)
    c = [torch.zeros_like(p, dtype=F16) for p in params] if copies else None
    for k in range(1, steps + 1):
        now = dict(kw) if k > start else {}
        aires.adamw(params, grads, m, v, step=k, lr=1e-2, seed=k, copies=c, **now)
    return params + [x for y in (m, v) for z in y for x in (z if bits == 8 else (z,))] + (c or [])


def same(a, b):
    assert len(a) == len(b) and all(equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_takes_any_number(bits):
    """A factor on the device gives the bits of the number; so does every other tensor of one
    value, whatever its type and place, and every number of any kind."""
    import numpy as np
    grads = [rand((33, 170), 3, BF16).cuda(), rand(300, 4, F16).cuda()]
    _, scale = aires.grad_norm(grads, max_norm=1.5)
    assert float(scale) < 0.1
    want = step(bits, grad_scale=float(scale))
    for x in (scale, scale.view(1), scale.cpu(), scale.double(), scale.cpu().double(), scale.view(1, 1).cpu(), np.float32(float(scale))):
        same(step(bits, grad_scale=x), want)
    want = step(bits, grad_scale=0.5)
    for x in (scale.new_full((), 0.5).to(BF16), torch.tensor(0.5, dtype=F16), np.float64(0.5), np.array(0.5)):
        same(step(bits, grad_scale=x), want)
    same(step(bits, grad_scale=torch.tensor(2)), step(bits, grad_scale=2))
    for bad in (torch.ones(2, device="cuda"), torch.ones(2), torch.empty(0, device="cuda"), "1", None):
        with pytest.raises((ValueError, TypeError)):
            step(bits, grad_scale=bad)
    for bad in (math.inf, math.nan, torch.tensor(math.nan), torch.tensor(math.inf, dtype=torch.float64).cuda()):
        with pytest.raises(aires.AiresError):
            step(bits, grad_scale=bad)


def moments(bits):
    return slice(3, 3 + (12 if bits == 8 else 6))


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_after_an_infinite_gradient(bits):
    """The norm's factor is 0: gradients count 0, and nothing that is kept becomes NaN."""
    shapes = [(33, 170), (300,), (4096,)]
    grads = [rand(s, 5 + i, t).cuda() for i, (s, t) in enumerate(zip(shapes, (BF16, F16, F32)))]
    bad = [g.clone() for g in grads]
    bad[0][3, 7], bad[2][4095] = math.inf, -math.inf
    norm, scale = aires.grad_norm(bad, max_norm=1.0)
    assert float(norm) == math.inf and float(scale) == 0
    nothing = [torch.zeros_like(g) for g in grads]

    def run(last, **kw):
        params = [rand(s, 1 + i).cuda() for i, s in enumerate(shapes)]
        m, v = aires.adamw_state(params, bits=bits)
        aires.adamw(params, grads, m, v, step=1, lr=1e-2, seed=1)
        aires.adamw(params, last, m, v, step=2, lr=1e-2, seed=2, **kw)
        return params + [x for y in (m, v) for z in y for x in (z if bits == 8 else (z,))]

    got = run(bad, grad_scale=scale)
    assert all(bool(x.float().isfinite().all()) for x in got)
    same(got, run(nothing))
    # of finite gradients: what a number gives; a NaN counts 0 too
    zero = torch.zeros((), device="cuda")
    same(run(grads, grad_scale=zero), run(grads, grad_scale=0.0))
    bad[1][0] = math.nan
    same(run(bad, grad_scale=zero), run(nothing))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("factor", [math.nan, math.inf, -math.inf])
def test_adamw_leaves_out_a_step_without_a_finite_factor(bits, factor):
    """Parameters and moments stay, bit for bit; copies receive the parameters."""
    scale = torch.full((), factor, device="cuda")
    one = step(bits, steps=1, copies=True)
    got = step(bits, steps=2, start=1, grad_scale=scale, copies=True)
    for a, b in zip(one[:-3], got[:-3]):
        assert bool((a.view(torch.uint8) == b.view(torch.uint8)).all())
    # (a step rounds its fp32 result to a parameter's type and to its copy's; here the copy
    # is the stored parameter's)
    for p, c in zip(got[:3], got[-3:]):
        assert bool((c == p.to(F16)).all())
    first = step(bits, steps=1, grad_scale=scale, copies=True)
    for p, c in zip(first[:3], first[-3:]):
        assert torch.equal(c, p.to(F16)) and bool(c.any())
    assert not any(bool(x.float().any()) for x in first[moments(bits)])


def test_adamw_leaves_out_a_step_after_a_nan():
    grads = [rand((33, 170), 3).cuda(), rand(300, 4).cuda()]
    params = [torch.ones_like(g) for g in grads]
    m, v = aires.adamw_state(params)
    grads[1][299] = math.nan
    _, scale = aires.grad_norm(grads, max_norm=1.0)
    aires.adamw(params, grads, m, v, step=1, lr=1e-2, grad_scale=scale)
    assert all(bool((p == 1).all()) for p in params) and not any(bool(x.any()) for x in m + v)
    grads[1][299] = 0
    _, scale = aires.grad_norm(grads, max_norm=1.0)
    aires.adamw(params, grads, m, v, step=1, lr=1e-2, grad_scale=scale)
    assert all(bool((p != 1).any()) and bool(p.isfinite().all()) for p in params)


# ------------------------------------------------------------- products' sums

@pytest.mark.parametrize("m", [16, 17, 300, 3600])
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
def test_product_of_sums_that_cancel(m, tiles, kind):
    """Each eight of k holds a large product and its negative, and six small ones, which are
    all that is left.  The sums of fp32 results and of up to 16 rows are fp32's: 128
    products, exact, in any order, with a whole step of the sum's size each.  Others may be
    off by 8 * 2^-13 of the largest product of each eight."""
    n, k = (3700, 272) if m == 3600 else (40, 656)
    g = torch.Generator(device="cuda").manual_seed(m)
    a = torch.randn((m, k), generator=g, device="cuda").to(F8).float()
    b = torch.randn((n, k), generator=g, device="cuda").to(F8).float()
    a[:, 0::8], a[:, 5::8], b[:, 0::8], b[:, 5::8] = 448, 448, 448, -448
    sa = torch.exp2(torch.randint(-3, 4, (m, -(-k // 128)), generator=g, device="cuda").float())
    sb = torch.exp2(torch.randint(-3, 4, (-(-n // 128) if tiles else n, -(-k // 128)), generator=g, device="cuda").float())
    got = aires.matmul_8bit((a.to(F8), sa), (b.to(F8), sb), out_dtype=kind).double()
    each = (sb.repeat_interleave(128, 0)[:n] if tiles else sb).repeat_interleave(128, 1)[:, :k].double()
    A, B = a.double() * sa.repeat_interleave(128, 1)[:, :k].double(), b.double() * each
    y = A @ B.t()
    tol = (256 + 6 + 16) * U * (A.abs() @ B.abs().t()) + rounded(y, kind)
    if kind != F32 and m > 16:
        for c in range(0, k, 8):  # the eight's largest product is that of two codes of 448
            tol += 8 * 2.0 ** -13 * A[:, c, None].abs() * B[None, :, c].abs()
    assert bool(((got - y).abs() <= tol).all()), float(((got - y).abs() / tol).max())


WAYS = [(5, 40, 300), (17, 40, 300), (100, 90, 4000), (300, 257, 400), (1800, 1800, 300), (3600, 3700, 272)]


@pytest.mark.parametrize("m,n,k", WAYS)
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("kind", [F32, BF16])
def test_product_with_an_infinite_scale(m, n, k, tiles, kind):
    """Infinities or NaNs in the rows and columns that the scales belong to, in others the
    bits as without them."""
    A = aires.quantize_8bit(rand((m, k), 1).cuda())
    B = aires.quantize_8bit(rand((n, k), 2).cuda(), tiles=tiles)
    clean = aires.matmul_8bit(A, B, out_dtype=kind)
    a, b = A[1].clone(), B[1].clone()
    a[3, -1], b[0, 0] = math.inf, math.inf
    got = aires.matmul_8bit((A[0], a), (B[0], b), out_dtype=kind)
    hit = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    hit[3], hit[:, :128 if tiles else 1] = True, True
    assert not bool(got[hit].isfinite().any()) and bool((got == clean)[~hit].all())


@pytest.mark.parametrize("m,n,k", WAYS)
@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("kind", [F32, BF16])
@pytest.mark.parametrize("low", [True, False])
def test_product_at_the_ends_of_its_scales_range(m, n, k, tiles, kind, low):
    """Scales that multiply to 2^-126 and 2^-125, and to 2^126 and 2^127 with codes that keep
    the results finite (k 2^-12 2^127 at most): as products of ordinary scales, times that power."""
    g = torch.Generator(device="cuda").manual_seed(m + k)
    steps = -(-k // 128)
    size = 1.0 if low else 2.0 ** -8                       # (codes of 2^-9 and 2^-8 and zeros)
    a = (torch.randn((m, k), generator=g, device="cuda") * size).clamp(-size * 448, size * 448).to(F8)
    b = (torch.randn((n, k), generator=g, device="cuda") * size).to(F8)
    if not low:
        a, b = (x.float().clamp(-2.0 ** -6, 2.0 ** -6).to(F8) for x in (a, b))
    sa = torch.exp2(torch.randint(0, 2, (m, steps), generator=g, device="cuda").float())
    sb = torch.ones((-(-n // 128) if tiles else n, steps), device="cuda")
    ea, eb = (-60, -66) if low else (60, 66)
    plain = aires.matmul_8bit((a, sa), (b, sb), out_dtype=kind).double()
    got = aires.matmul_8bit((a, sa * 2.0 ** ea), (b, sb * 2.0 ** eb), out_dtype=kind).double()
    want = plain * 2.0 ** (ea + eb)
    assert bool(want.abs().amax() < 3e38)
    # the same bits but for what falls below a type's normal numbers in each of the blocks' sums and the result
    least = 2.0 ** -149 if kind == F32 else 2.0 ** -133
    assert bool(((got - want).abs() <= (steps + 16) * 2.0 ** -149 + least).all())


# ------------------------------------------------- gradients far from zero

FAR = [(F32, 0.0), (F32, 1e3), (F32, -1e5), (F32, 2.0 ** 24), (BF16, 3e4), (BF16, -3e38), (F16, -6e4)]


@pytest.mark.parametrize("t,v", [(5, 6), (40, 30), (40, 100), (9, 500), (30, 700), (600, 2100), (3, 30011)])
@pytest.mark.parametrize("kind,offset", FAR)
def test_gradient_of_scores_far_from_zero(t, v, kind, offset):
    """Against p from 64 bits.  With what lse's rounding leaves, p is off by 3 U |log p| + 8 U
    of itself (the difference, its product with log2 e, the exponential) and by the sum
    that the forward pass made; without, by |lse| U more."""
    z = (3 * rand((t, v), t + v) + offset).to(kind)
    z[0] = torch.finfo(kind).min if offset <= 0 else torch.finfo(kind).max
    z[1, : v // 2] = -math.inf
    z[2] = -math.inf
    labels = torch.randint(-1, v, (t,), generator=torch.Generator().manual_seed(t))
    a, b = rand(t, 5), rand(t, 6)
    # (64 bits lose the logarithm of a sum next to 3e38 too: all from the row's maximum)
    m = z.double().amax(1)
    some = m > -math.inf
    m = torch.where(some, m, torch.zeros(()).double())
    log_s, _, H, lp, p = logp_ref(z.double() - m[:, None], labels)
    lse, log_s = m + log_s, torch.where(some, log_s, torch.zeros(()).double())
    r = aires.log_probs(z.cuda(), labels.cuda(), rest=True)
    plain = aires.log_probs(z.cuda(), labels.cuda())
    assert plain.lse_rest is None and equal(plain.lse, r.lse) and equal(plain.entropy, r.entropy) and equal(plain.logp, r.logp)
    base, _ = logp_tolerance(z.double() - m[:, None], p)
    near((r.lse.double().cpu() - m) + r.lse_rest.double().cpu(), torch.where(some, log_s, lse), base + 2 * U * log_s.abs(),
         "lse and its rest, from the maximum")
    assert float(r.lse_rest[2]) == 0

    d = torch.where(p > 0, lp, torch.zeros(()).double())
    there = (labels >= 0) & some
    A = torch.where(there, a, torch.zeros(())).double()[:, None]
    B, h = b.double()[:, None], H.float()
    hot = torch.zeros(t, v, dtype=torch.float64).scatter_(1, labels.clamp(0, v - 1)[:, None], there.double()[:, None])
    want = A * hot - p * (A + B * (d + h.double()[:, None]))
    size = A.abs() + B.abs() * (d.abs() + H[:, None])
    off = (base + 2 * U * log_s.abs())[:, None]           # of lse and its rest
    rest = r.lse_rest.double().cpu().abs()[:, None]

    def tolerance(off):
        return (p * (size * (torch.expm1(off) * 1.01 + (3 * d.abs() + 14 + 3 * rest) * U) + B.abs() * (off + 4 * U * (d.abs() + H[:, None] + rest)))
                + U * (A.abs() * hot + p * size))

    args = dict(dlogp=a.cuda(), dentropy=b.cuda())
    got = aires.log_probs_backward(z.cuda(), labels.cuda(), r.lse, h.cuda(), lse_rest=r.lse_rest, **args)
    assert got.dtype == kind
    near(got, want, tolerance(off) + rounded(want, kind), "dZ")
    wide = aires.log_probs_backward(z.cuda(), labels.cuda(), r.lse, h.cuda(), lse_rest=r.lse_rest, dz_dtype=F32, **args)
    near(wide, want, tolerance(off) + rounded(want, F32), "dZ in fp32")
    own = z.cuda()
    aires.log_probs_backward(own, labels.cuda(), r.lse, h.cuda(), lse_rest=r.lse_rest, out=own, **args)
    assert equal(own, got)
    if abs(offset) <= 1e5:  # lse alone: the row at the end of its type's range (the first) has lost log sum
        lone = aires.log_probs_backward(z.cuda(), labels.cuda(), r.lse, h.cuda(), dz_dtype=F32, **args)
        more = off + (U * lse.abs().nan_to_num(posinf=0, neginf=0))[:, None]
        near(lone[1:], want[1:], (tolerance(more) + rounded(want, F32))[1:], "dZ of lse alone")


def test_what_the_rounding_of_lse_leaves():
    z = rand((20, 77), 1).cuda()
    r = aires.log_probs(z, top=3, rest=True)
    assert r.lse_rest.shape == (20,) and r.lse_rest.dtype == F32 and r.top_index.shape == (20, 3)
    z[3, 5], z[4, 6] = math.nan, math.inf
    r = aires.log_probs(z, rest=True)
    assert bool(r.lse[3:5].isnan().all()) and bool(r.lse_rest.isfinite().all())
    dz = aires.log_probs_backward(z, None, r.lse, r.entropy, lse_rest=r.lse_rest, dentropy=r.lse_rest + 1)
    assert bool(dz[3:5].isnan().all()) and bool(dz[:3].isfinite().all()) and bool(dz[5:].isfinite().all())
    for bad in (r.lse_rest[:3], r.lse_rest.double(), r.lse_rest.cpu()):
        with pytest.raises((ValueError, TypeError)):
            aires.log_probs_backward(z, None, r.lse, lse_rest=bad)
