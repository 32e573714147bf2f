"""Every kernel that the library holds for the layers' calls is launched by a call (GPU)."""
import os
import re

import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from paper_2507_02006_amd import _binding as B_  # noqa: E402
from test_gpu_layers import BF16, F8, F16, F32  # noqa: E402
from test_kernel_resources import code_objects, kernels  # noqa: E402

pytestmark = pytest.mark.gpu

OURS = re.compile(r"^k_(rms_|quantize|tiles8|join8|rows8|zero8|pack8|logp_|grad_(norm|squares|scale)$)")


def built():
    """(name, template arguments) of the layers' kernels in the library."""
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


def norms():
    for n in (5, 40, 100, 200, 400, 800, 1800, 3000, 8000, 12000, 17000, 0):
        for a, b in ((F32, F32), (BF16, BF16), (F16, F16), (F32, BF16)):
            x, r = torch.zeros(70, n, dtype=a, device="cuda"), torch.zeros(70, n, dtype=b, device="cuda")
            for residual in (None, r):
                for out in (b, F8):
                    _, _, q = aires.rms_norm(x, residual=residual, out_dtype=out)
                aires.rms_norm_backward(r, x, q, dS=residual)


def codes():
    for x in [torch.zeros(300, n, dtype=t, device="cuda") for n in (5, 300) for t in (F32, BF16, F16)]:
        for tiles in (False, True):
            for order in ("rows", "columns", "both"):
                aires.quantize_8bit(x, tiles=tiles, order=order)


def products():
    for tiles in (False, True):
        for m, n, k in ((3, 40, 256), (3, 40, 255), (100, 40, 255), (181, 38, 17328), (100, 100, 2048), (1792, 1800, 128),
                        (3900, 3600, 128), (30, 20, 0)):
            A, B = (aires.quantize_8bit(torch.zeros(r, k, device="cuda"), tiles=t) for r, t in ((m, False), (n, tiles)))
            for out in (F32, BF16):
                aires.matmul_8bit(A, B, out_dtype=out)


def scores():
    for kind in (F32, BF16, F16):
        for v in (5, 50, 100, 200, 400, 600, 30000):
            z = torch.zeros(30, v, dtype=kind, device="cuda")
            y = torch.zeros(30, dtype=torch.int64, device="cuda")
            for top in (0, 1, 3, 20):
                r = aires.log_probs(z, y, top=min(top, v))
            for out in (kind, F16 if kind == F32 else F32):
                aires.log_probs_backward(z, y, r.lse, dlogp=r.logp, dz_dtype=out)


def gradients():
    for n in (300, 1 << 24):
        g = [torch.zeros(n, device="cuda")]
        aires.grad_norm(g)
        aires.clip_grads(g, 1.0)


def test_every_kernel_runs():
    from torch.profiler import ProfilerActivity, profile
    want = built()
    assert len(want) > 200

    def calls():
        for f in (norms, codes, products, scores, gradients):
            f()
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
