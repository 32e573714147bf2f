"""Layer norm, cross entropy and AdamW at the edges of what they take (GPU).

U = 2^-24 is the unit roundoff of fp32: a sum of any order, in chains of at
most c additions, is off by c U times the sum of magnitudes.
"""
import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def gen(seed):
    return torch.Generator().manual_seed(seed)


# -------------------------------------------------------------- layer norm

@pytest.mark.parametrize("m", [1, 4, 300, 70001])
def test_layer_norm_statistics_of_rows_without_columns(m):
    X = torch.empty(m, 0, device="cuda")
    held = torch.full((2 * m + 64,), float("nan"), device="cuda")  # what the results' memory may hold before
    del held
    for eps in (1e-5, 0.25):
        Y, mean, rstd = aires.layer_norm(X, eps=eps)
        assert Y.shape == (m, 0) and mean.shape == rstd.shape == (m,)
        assert not mean.any() and torch.allclose(rstd, torch.full_like(rstd, eps ** -0.5), rtol=4 * U, atol=0)


def test_layer_norm_gradients_of_more_columns_than_a_launch_has_threads_for():
    n = (1 << 27) + 37
    g = torch.Generator(device="cuda").manual_seed(1)
    X, dY = (torch.randint(-4, 5, (2, n), generator=g, device="cuda", dtype=torch.int8).to(F16) for _ in range(2))
    mean, rstd = torch.tensor([0.5, 0.0], device="cuda"), torch.tensor([0.25, 2.0], device="cuda")
    dX, dgamma, dbeta = aires.layer_norm_backward(dY, X, mean, rstd, need_dx=False)  # (small numbers: all exact)
    assert dX is None
    assert torch.equal(dbeta, dY[0].float() + dY[1].float())
    assert torch.equal(dgamma, dY[0].float() * ((X[0].float() - 0.5) * 0.25) + dY[1].float() * (X[1].float() * 2))
    none = torch.empty(0, n, dtype=F16, device="cuda")
    for t in aires.layer_norm_backward(none, none, mean[:0], rstd[:0], need_dx=False)[1:]:
        assert t.shape == (n,) and not t.any()


# ----------------------------------------------------------- cross entropy

@pytest.mark.parametrize("dt", [F32, BF16, F16])
@pytest.mark.parametrize("t,d,v", [(300, 64, 40), (70, 800, 20), (20, 131, 3000), (64, 256, 3000), (1, 512, 5000),
                                   (500, 96, 2000), (2100, 72, 300), (140, 256, 60013)])
def test_loss_of_rows_whose_label_dominates(t, d, v, dt):
    """Scores that are multiples of 1/16 of up to eight times the columns, exact
    in every type and order; the label's is the largest, and one other is k, 1 to 8,
    below it or all are far below.  The loss is then log(1 + e^-k + ...) with
    nothing lost to the scores' size, and never negative."""
    g = gen(t + d + v)
    W = torch.randint(0, 2, (v, d), generator=g).mul(2).sub(1).double()
    W[v // 2] = W[3]
    W[v // 2, 0] = 0  # next to class 3: k less
    y = torch.randint(0, v, (t,), generator=g)
    y[::3] = 3
    k = torch.randint(16, 128, (t,), generator=g).double() / 16
    H = W[y] * k[:, None]
    z = H @ W.t()
    top = z.amax(1, keepdim=True)
    assert bool((z.abs() < 2 ** 14).all())
    total = torch.exp(z - top).sum(1)
    want = (top[:, 0] - z[torch.arange(t), y]) + torch.log1p((total - 1).clamp(min=0))
    H, W = H.to(dt).cuda(), W.to(dt).cuda()
    for grads in (False, True):
        got = aires.linear_xent(H, W, y.cuda(), grads=grads)
        rows = got.row_loss.double().cpu()
        # a sum of at least 1 in chains of at most 256 additions, exponentials and a logarithm in fp32
        tol = 256 * U * (1 + want)
        assert bool((rows >= 0).all()), float(rows.min())
        assert bool(((rows - want).abs() <= tol).all()), float(((rows - want).abs() / tol).max())
        assert abs(float(got.loss) - float(want.mean())) <= 256 * U * (1 + float(want.mean()))


def test_small_probabilities_in_half_precision():
    """dW of classes whose probability is below 2^-24 with a large gradient
    scale: they keep all the bits that an fp16 result has."""
    t, d, v, scale = 100, 64, 300, 2.0 ** 15
    H = torch.ones(t, d)
    a = torch.arange(v).double() * 2.0 ** -10 + 17.0 / d  # scores of -17 to -36, exact in fp16 and in any order
    a = -(a * 2 ** 10).round() / 2 ** 10
    a[0] = 0
    W = a[:, None].expand(v, d).contiguous()
    assert torch.equal(W.half().double(), W)
    y = torch.zeros(t, dtype=torch.int64)
    got = aires.linear_xent(H.half().cuda(), W.half().cuda(), y.cuda(), reduction="sum", grad_scale=scale)
    p = torch.softmax(d * a, 0)
    want = (t * scale * p)[1:, None]
    some = p[1:] >= 2.0 ** -29  # (below them dz is not a normal number of 16 bits)
    assert int(some.sum()) > 40
    # dz and the result are rounded to 11 bits; the exponent's argument is off by 4 U of 36 log2 e
    tol = (2 * 2.0 ** -11 + 4 * 52 * U + 64 * U) * want
    assert bool(((got.dW.double().cpu()[1:] - want).abs() <= tol)[some].all())


# --------------------------------------------------------- tensors of torch's

def test_tensors_that_are_written_count_a_version():
    """A backward pass that kept a value from before raises instead of reading the new one."""
    p = [torch.ones(300, device="cuda", requires_grad=True), torch.ones(5, 7, device="cuda")]
    q = [torch.full_like(x, 0.1) for x in p]
    copies = [torch.empty(300, dtype=BF16, device="cuda"), None]
    for bits in (32, 8):
        M, V = aires.adamw_state(p, bits=bits)
        all_of = [*p, copies[0], *(y for x in (M + V) for y in (x if bits == 8 else (x,)))]
        kept = (p[0] * p[0]).sum()
        before, untouched = [x._version for x in all_of], [x._version for x in q]
        aires.adamw(p, q, M, V, step=1, lr=0.1, copies=copies)
        assert all(x._version > b for x, b in zip(all_of, before))
        assert [x._version for x in q] == untouched
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.backward()
    X, out = torch.randn(4, 6, device="cuda"), torch.empty(4, 6, device="cuda")
    before = out._version, X._version
    aires.layer_norm(X, out=out)
    assert out._version > before[0] and X._version == before[1]
    with torch.inference_mode():  # (no versions there)
        x = [torch.ones(8, device="cuda")]
        M, V = aires.adamw_state(x)
        aires.adamw(x, [torch.ones(8, device="cuda")], M, V, step=1, lr=0.5, weight_decay=0.0)
        aires.layer_norm(X, out=torch.empty(4, 6, device="cuda"))
    assert torch.allclose(x[0], torch.full((8,), 0.5, device="cuda"))


@pytest.mark.parametrize("what", ["layer_norm", "layer_norm_backward", "linear_xent", "adamw", "adamw_8"])
def test_inputs_released_before_another_stream_reads_them(what):
    """The call is behind other work on its stream when its inputs' last
    references go; their memory is not handed out before it has run."""
    m, n = 2048, 640
    x, gamma = torch.randn(m, n, generator=gen(1)).cuda(), torch.ones(n, device="cuda")
    W, y = torch.randn(300, n, generator=gen(2)).cuda(), torch.arange(m, device="cuda") % 300
    _, mean, rstd = aires.layer_norm(x, gamma)
    p, bits = [torch.ones(m, n, device="cuda")], 8 if what == "adamw_8" else 32
    M, V = aires.adamw_state(p, bits=bits)

    def call(X, **kw):
        if what == "layer_norm":
            return list(aires.layer_norm(X, gamma, **kw))
        if what == "layer_norm_backward":
            return list(aires.layer_norm_backward(X, x, mean, rstd, gamma, **kw))
        if what == "linear_xent":
            r = aires.linear_xent(X, W, y, **kw)
            return [r.loss, r.row_loss, r.dH, r.dW]
        # (any sequence will do)
        aires.adamw(torch.nn.ParameterList(p), torch.nn.ParameterList([X]), M, V, step=1, lr=0.5, **kw)
        return [p[0]]

    def reset():
        p[0].fill_(1.0)
        for state in (M, V):
            for t in (state[0] if bits == 8 else state):
                t.zero_()

    reset()
    want = [t.clone() for t in call(x.clone())]
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for stream in (s, s.cuda_stream):
        X = x.clone()
        reset()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(20):
                big @ big
        got = call(X, stream=stream)
        del X
        over = [torch.full((m, n), float("nan"), device="cuda") for _ in range(3)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        del over
