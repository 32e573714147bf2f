"""The layers' calls where their arguments end (GPU): no rows, factors and scales that are
not ordinary numbers, scores far from zero."""
import math

import pytest

torch = pytest.importorskip("torch")
import paper_2507_02006_amd as aires  # noqa: E402
from test_gpu_layers import BF16, F16, F32, F8, U, equal, near, rand, rounded  # noqa: E402,F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("v", [5, 300, 2049, 100000])
def test_log_probs_of_no_rows(v):
    z, labels = torch.empty(0, v, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    for top in (0, 1, 5):
        r = aires.log_probs(z, labels, top=top)
        assert r.logp.shape == r.entropy.shape == r.lse.shape == (0,)
        assert top == 0 or r.top_index.shape == r.top_logp.shape == (0, top)
    assert aires.log_probs_backward(z, labels, r.lse, r.entropy, dlogp=r.logp, dentropy=r.entropy).shape == (0, v)
