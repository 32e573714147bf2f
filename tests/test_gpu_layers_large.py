"""The layers' calls on arrays whose places pass 32 bits (GPU): rows far apart in
memory, and many rows, each against the same call on copies of a few of them."""
import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from test_gpu_layers import BF16, F8, F32, rand  # noqa: E402

pytestmark = pytest.mark.gpu

FAR = (1 << 31) + 24  # values from one row to the next: 4 GB of 16-bit ones


def far(m, n, dtype, value=None):
    """m x n with rows FAR values apart."""
    x = torch.empty((m - 1) * FAR + n, dtype=dtype, device="cuda").as_strided((m, n), (FAR, 1))
    if value is not None:
        x.copy_(value)
    return x


def words(x):
    return x.contiguous().view(torch.uint8)


@pytest.mark.parametrize("n", [200, 4100, 17000])
def test_norm_of_rows_far_apart(n):
    x, r, dy = (rand((3, n), k, BF16).cuda() for k in (1, 2, 3))
    gamma = rand((n,), 4).cuda()
    X, R = far(3, n, BF16, x), far(3, n, BF16, r)
    Y, S, q = aires.rms_norm(x, gamma, residual=r)
    out = far(3, n, BF16)
    Y2, S2, q2 = aires.rms_norm(X, gamma, residual=R, sum_out=R, out=out)
    assert torch.equal(Y, Y2) and torch.equal(S, S2) and torch.equal(q, q2)
    codes, scales = aires.rms_norm(x, gamma, out_dtype=F8)[0]
    codes2, scales2 = aires.rms_norm(X, gamma, out_dtype=F8)[0]
    assert torch.equal(words(codes), words(codes2)) and torch.equal(scales, scales2)
    X.copy_(dy)
    want = aires.rms_norm_backward(dy, S, q, gamma, dS=r)
    have = aires.rms_norm_backward(X, R, q, gamma, dS=r)
    assert all(torch.equal(a, b) for a, b in zip(want, have))


@pytest.mark.parametrize("tiles", [False, True])
def test_codes_of_rows_far_apart(tiles):
    x = rand((3, 300), 1, BF16).cuda()
    X = far(3, 300, BF16, x)
    for order in ("rows", "columns", "both"):
        want, have = (aires.quantize_8bit(v, tiles=tiles, order=order) for v in (x, X))
        want, have = ([want], [have]) if order != "both" else (want, have)
        for a, b in zip(want, have):
            assert torch.equal(words(a[0]), words(b[0])) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("m,apart", [(3, FAR), (40, FAR // 8)])
def test_product_with_results_far_apart(m, apart):
    """Rows of Y far apart, in one share of k and (m = 40) in several."""
    A = aires.quantize_8bit(rand((m, 4096), 1, BF16).cuda())
    B = aires.quantize_8bit(rand((72, 4096), 2, BF16).cuda(), tiles=True)
    want = aires.matmul_8bit(A, B)
    out = torch.empty((m - 1) * apart + 72, dtype=BF16, device="cuda").as_strided((m, 72), (apart, 1))
    aires.matmul_8bit(A, B, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("m,n,k", [(530, 40, 1 << 23), (8, 600, 1 << 23)])
def test_product_of_operands_past_four_gigabytes(m, n, k):
    """Codes that are 0 but in the last blocks of the last rows: sums of a few products."""
    def operand(rows, seed):
        codes = torch.zeros((rows, k), dtype=torch.uint8, device="cuda").view(F8)
        scales = torch.ones((rows, k // 128), device="cuda")
        codes[:, -300:] = rand((rows, 300), seed).cuda().to(F8)
        return codes, scales

    A, B = operand(m, 1), operand(n, 2)
    Y = aires.matmul_8bit(A, B, out_dtype=F32)
    a, b = (x[0][:, -300:].float().double() for x in (A, B))
    want = a @ b.t()
    # 300 products added in fp32: at most 300 sums, each rounded or cut to 24 bits of at
    # most the products' sizes together
    assert ((Y.double() - want).abs() <= 300 * 2.0 ** -23 * (a.abs() @ b.abs().t())).all()


@pytest.mark.parametrize("v,top", [(5, 3), (300, 3), (1500, 3), (40000, 3), (40000, 0)])
def test_log_probs_of_rows_far_apart(v, top):
    z = rand((3, v), 1, BF16).cuda()
    Z = far(3, v, BF16, z)
    labels = torch.tensor([0, v - 1, v // 2], device="cuda")
    a, b = aires.log_probs(z, labels, top=top), aires.log_probs(Z, labels, top=top)
    for name in ("logp", "entropy", "lse", "top_logp", "top_index"):
        x, y = getattr(a, name), getattr(b, name)
        assert x is y is None or torch.equal(x, y), name
    ones = torch.ones(3, device="cuda")
    want = aires.log_probs_backward(z, labels, a.lse, a.entropy, dlogp=ones, dentropy=ones)
    have = aires.log_probs_backward(Z, labels, b.lse, b.entropy, dlogp=ones, dentropy=ones, out=Z)
    assert torch.equal(want, have) and have.data_ptr() == Z.data_ptr()


def test_many_rows():
    """More rows than a launch has threads' worth of, the last ones against a call of their own."""
    m = (1 << 25) + 1000
    x = torch.zeros((m, 96), dtype=BF16, device="cuda")
    x[-2000:] = rand((2000, 96), 1, BF16).cuda()
    gamma = rand((96,), 2).cuda()
    Y, _, q = aires.rms_norm(x, gamma)
    Y2, _, q2 = aires.rms_norm(x[-2000:], gamma)
    assert torch.equal(Y[-2000:], Y2) and torch.equal(q[-2000:], q2)
    dx, dg = aires.rms_norm_backward(x, x, q, gamma)
    dx2, dg2 = aires.rms_norm_backward(x[-2000:], x[-2000:], q2, gamma)
    assert torch.equal(dx[-2000:], dx2)
    # zeros add nothing; both sums are of 2000 products at most, in other orders
    size = (x[-2000:].double() ** 2 * q2.double()[:, None]).sum(0)
    assert ((dg.double() - dg2.double()).abs() <= 2 * 2004 * 2.0 ** -24 * size).all()
    codes, scales = aires.quantize_8bit(x)
    codes2, scales2 = aires.quantize_8bit(x[-2000:])
    assert torch.equal(words(codes[-2000:]), words(codes2)) and torch.equal(scales[-2000:], scales2)
    del Y, dx, codes, scales
    a, b = aires.log_probs(x, top=2), aires.log_probs(x[-2000:], top=2)
    assert torch.equal(a.lse[-2000:], b.lse) and torch.equal(a.top_index[-2000:], b.top_index)
    norm, scale = aires.grad_norm([x], max_norm=1.0)
    want = x[-2000:].double().pow(2).sum().sqrt()
    assert abs(float(norm) - float(want)) <= 2.0 ** -23 * float(want)
    aires.clip_grads([x], 1.0)
    assert abs(float(aires.grad_norm([x])[0]) - 1) <= 2.0 ** -8


def test_many_long_rows():
    """More rows of scores than one launch takes, a workgroup or a wavefront each."""
    t, v = (1 << 23) + 77, 520
    z = torch.zeros((t, v), dtype=BF16, device="cuda")
    z[-500:] = rand((500, v), 1, BF16).cuda()
    labels = torch.full((t,), v - 1, device="cuda")
    a, b = aires.log_probs(z, labels, top=2), aires.log_probs(z[-500:], labels[-500:], top=2)
    for name in ("logp", "entropy", "lse", "top_logp", "top_index"):
        assert torch.equal(getattr(a, name)[-500:], getattr(b, name)), name
    assert (a.lse[:-500] == a.lse[0]).all() and (a.top_index[:-500] == torch.tensor([0, 1], device="cuda")).all()
    ones = torch.ones(t, device="cuda")
    dz = aires.log_probs_backward(z, labels, a.lse, dlogp=ones)
    dz2 = aires.log_probs_backward(z[-500:], labels[-500:], b.lse, dlogp=ones[-500:])
    assert torch.equal(dz[-500:], dz2)
