"""Values at the edges of the product of level bytes: what is not finite, and what nearly cancels."""
import math

import numpy as np
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


def exact(act, y):
    if act == "gelu":
        return np.array([0.5 * v * math.erfc(-v / math.sqrt(2)) for v in y])
    if act == "gelu_tanh":
        return y / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    return y / (1 + np.exp(-y))


@pytest.mark.parametrize("act", ["gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("rows", [1, 513])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_negative_tails_keep_their_relative_precision(mpq, cuda, act, rows, dtype):
    """Arguments from -8 to -3, where the results fall to 5e-15: the product is 0 and the bias is the argument.
    Tolerance, relative to the result.  GELU: the argument of erfc carries two roundings of 2^-24, which move the result by
    z^2 times as much (f erfc(z) changes by 2 z^2 + 1 per relative change of z, z^2 <= 32: 66 * 2^-23), erfc itself is good
    to some units, 2^-21, and two products, 2^-23: under 2^-16.  The other two: an exponential of at most 50 whose argument
    carries up to eight roundings of 2^-24 (50 * 8 * 2^-24 = 2^-15.4) and whose own error is 60 units (2^-18), and a
    quotient of 2 units: under 2^-15.  Then the last rounding."""
    f = np.linspace(-8, -3, 2177 if rows > 1 else 300).astype(np.float32)
    n, k = len(f), 16
    flat = lambda count, v: mpq.Levels(torch.full((count, k), v, dtype=torch.uint8, device=cuda), torch.zeros(count, device=cuda),       # noqa: E731
                                       torch.full((count,), v * k, dtype=torch.int32, device=cuda), 8, k)
    got = mpq.linear_levels(flat(rows, 3), flat(n, 200), bias=torch.from_numpy(f).to(cuda), act=act, dtype=dtype).double().cpu().numpy()
    want = exact(act, f.astype(np.float64))
    rel = (2.0 ** -16 if act == "gelu" else 2.0 ** -15) + (2.0 ** -8 if dtype is torch.bfloat16 else 0.0)
    assert (np.abs(got - want) <= rel * np.abs(want)).all(), np.abs(got / want - 1).max()
