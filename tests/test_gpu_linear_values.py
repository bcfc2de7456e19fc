"""Values at the edges of the product of level bytes: what is not finite, and what nearly cancels."""
import pytest
import torch

from tests.test_gpu_linear_levels import operand

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("m,n", [(5, 30), (40, 300), (513, 2177)])        # both forms, the small one with k in parts
def test_non_finite_ranges_stay_visible_under_every_activation(mpq, cuda, act, m, n):
    a, _, _ = operand(mpq, cuda, m, 512, 8, 4)
    w, _, _ = operand(mpq, cuda, n, 512, 8, 5)
    ref = mpq.linear_levels(a, w, act=act)
    a.scale[3] = float("nan")
    w.scale[7] = float("nan")
    got = mpq.linear_levels(a, w, act=act)
    assert torch.isnan(got[3]).all() and torch.isnan(got[:, 7]).all()
    keep_r, keep_c = [i for i in range(m) if i != 3], [i for i in range(n) if i != 7]
    assert torch.equal(got[keep_r][:, keep_c], ref[keep_r][:, keep_c])
