"""The layers' calls at sizes that take their largest tiles and longest lists (GPU), against
64 bits on the device.  Tolerances are those of test_gpu_layers.py."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from test_gpu_layers import BF16, F16, F32, F8, U, logp_ref, logp_tolerance, near, rand, rounded  # noqa: E402

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


# ------------------------------------------------------------------ products

def codes(m, k, tiles, seed):
    """Codes of any size and scales that differ from block to block, by up to 2^6."""
    g = gen(seed)
    c = (16 * torch.randn((m, k), generator=g, device="cuda")).to(F8)
    rows = -(-m // 128) if tiles else m
    return c, torch.exp2(6 * torch.rand((rows, -(-k // 128)), generator=g, device="cuda") - 3)


def meant(held):
    c, s = held
    m, k = c.shape
    s = (s.repeat_interleave(128, 0)[:m] if s.shape[0] != m else s).double()
    return c.float().double() * s.repeat_interleave(128, 1)[:, :k]


# a tile's rows and columns, and how many workgroups share k, of a product of these sizes:
# 256 x 256 with B in tiles and 16-bit results, 128 x 128 otherwise
LARGE = [(3600, 3700, 1205, True, (BF16, F16)), (3600, 3700, 1200, True, (BF16, F16)), (3601, 3699, 2320, True, (BF16,)),
         (1800, 1800, 1200, True, (F32, BF16, F16)), (1800, 1800, 1205, False, (F32, BF16, F16)),
         (3600, 3700, 1205, False, (F32, BF16)), (3600, 3700, 656, True, (F32,)),
         (1000, 520, 20000, True, (F32, BF16, F16)), (1000, 520, 20013, False, (F32, BF16)), (700, 700, 17 * 1024 + 3, True, (F32, F16)),
         (2048, 1024, 5 * 128 + 16, False, (F32, BF16))]


@pytest.mark.parametrize("m,n,k,tiles,kinds", LARGE, ids=str)
def test_product_in_large_tiles(m, n, k, tiles, kinds):
    """More than one group of four steps' scales, k that ends inside a step, shares of k that
    are joined; every block with scales of its own."""
    A, B = codes(m, k, False, m + k), codes(n, k, tiles, n + k)
    a, b = meant(A), meant(B)
    y = a @ b.t()
    a, b = a.abs(), b.abs()
    sums = (256 + -(-k // 128) + 16) * U * (a @ b.t())
    eights = None
    for kind in kinds:
        # (a power of two brings results into fp16's range, and is all that it changes)
        by = 2.0 ** -16 if kind == F16 else 1.0
        tol = by * sums + rounded(by * y, kind)
        if kind != F32:
            if eights is None:
                eights = torch.zeros_like(y)
                for c in range(0, k, 8):
                    most = a[:, c, None] * b[None, :, c]
                    for i in range(c + 1, min(c + 8, k)):
                        most = torch.maximum(most, a[:, i, None] * b[None, :, i])
                    eights += 8 * 2.0 ** -13 * most
            tol = tol + by * eights
        got = aires.matmul_8bit((A[0], by * A[1]), B, out_dtype=kind)
        assert got.dtype == kind
        bad = ~((got.double() - by * y).abs() <= tol)
        assert not bool(bad.any()), (kind, int(bad.sum()), bad.nonzero()[0].tolist())


# ------------------------------------------------------------- log probabilities

@pytest.mark.parametrize("t,v", [(2100, 2500), (2048, 9001), (2049, 16384), (2048, 2049)])
@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("order", ["any", "rising", "falling", "equal"])
def test_log_probs_of_many_long_rows(t, v, kind, order):
    """Rows that a wavefront streams by itself, lists that overflow many times over a row."""
    g = gen(t + v)
    z = 3 * torch.randn((t, v), generator=g, device="cuda")
    if order == "equal":
        z = (z / 2).round() * 2 + 0.0
    z = z.to(kind)
    if order in ("rising", "falling"):
        z = z.sort(1, descending=order == "falling")[0]
    else:
        z.masked_fill_(torch.rand((t, v), generator=g, device="cuda") < 0.2, -math.inf)
    z[0], z[1], z[1, v - 1] = -math.inf, -math.inf, 1
    labels = torch.randint(-1, v + 1, (t,), generator=g, device="cuda")
    lse, logp, H, lp, p = logp_ref(z, labels)
    base, ent = logp_tolerance(z, p)
    # a maximum that rises with every chunk brings the sums to the new one as often
    more = 8 * U * (1 + H) * (v // 512 + 1) if order == "rising" else torch.zeros_like(H)
    best = torch.sort(z.float(), dim=1, descending=True, stable=True)[1]
    for top in (0, 1, 5, 20, 64):
        r = aires.log_probs(z, labels, top=top)
        near(r.lse, lse, base + more + 2 * U * lse.abs(), "lse")
        near(r.entropy, H, ent + more * (1 + H) + 4 * U * (H + 1), "entropy")
        near(r.logp, logp, base + more + 4 * U * logp.abs(), "logp")
        if top:
            assert bool((r.top_index == best[:, :top]).all()), top
            want = lp.gather(1, best[:, :top])
            near(r.top_logp, want, (base + more)[:, None] + 4 * U * want.abs().nan_to_num(0, 0, 0), "top")


# ------------------------------------------------------------------- clipping

@pytest.mark.parametrize("kind", [F32, BF16, F16])
@pytest.mark.parametrize("sizes", [[40003] * 300, [9000001, 5, 70000, 1], [3 << 20] * 5 + [7] * 200], ids=lambda s: "%d tensors" % len(s))
def test_clipping_of_many_partial_sums(kind, sizes):
    """More than 1024 partial sums (a launch of their own adds them), in one table of tensors
    and in several: every value, in place and to other types."""
    grads = [rand(n, i + n, kind).cuda() for i, n in enumerate(sizes)]
    want = math.sqrt(math.fsum(float(g.double().square().sum()) for g in grads))
    most = want / 3
    norm, scale = aires.grad_norm(grads, max_norm=most)
    assert abs(float(norm) - want) <= 1.01 * U * want and abs(float(scale) - 1 / 3) <= 1.01 * U
    for out in (kind, F32, BF16):
        outs = [torch.full(g.shape, 9.0, dtype=out, device="cuda") for g in grads]
        keep = [g.clone() for g in grads]
        assert float(aires.clip_grads(grads, most, out=outs)) == float(norm)
        for g, k, o in zip(grads, keep, outs):
            assert bool((g == k).all()) and bool((o == (g.float() * scale).to(out)).all())
    outs = [torch.empty_like(g) for g in grads]
    aires.clip_grads(grads, 2 * want, out=outs)
    assert all(bool((o == g).all()) for g, o in zip(grads, outs))
    mine = [g.clone() for g in grads]
    assert float(aires.clip_grads(mine, most)) == float(norm)
    assert all(bool((m == (g.float() * scale).to(kind)).all()) for g, m in zip(grads, mine))
    aires.clip_grads(mine, want)
    assert all(bool((m == (g.float() * scale).to(kind)).all()) for g, m in zip(grads, mine))
