"""Product of level bytes with adapters that hold infinities."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_adapted import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens,ids,n", [([3, 2, 4], [0, 1, 2], 300), ([40], [1], 130), ([600], [1], 1601), ([300, 300, 100], [0, 1, 2], 1601), ([520, 1, 300], [1, -1, 1], 777)])
def test_infinities_in_up_are_infinities(mpq, cuda, lens, ids, n, dtype):
    """Whatever the number of rows: z times an infinity is one of z's sign, and NaN where two meet or z is 0."""
    for rank in (16, 64):
        c = Case(mpq, cuda, lens, ids, n, 64, rank, dtype, seed=rank)
        plain = {out: c.run(dtype=out) for out in (torch.float32, torch.float16, torch.bfloat16)}
        c.up[1, 7, 3] = math.inf
        c.up[1, 9, 0] = -math.inf
        c.up[1, 40, 2], c.up[1, 40, 5] = math.inf, math.inf    # of one sign or of two, by the row
        c.up[1, n - 1, 15] = math.inf
        c.low = mpq.adapters(c.down.to(cuda), c.up.to(cuda), c.factor.to(cuda))
        with np.errstate(invalid="ignore"):
            want = sum(c.sums()[:2])
        for out, ref in plain.items():
            got = c.run(dtype=out)
            whole = np.isfinite(want)
            assert (~whole).sum() == 4 * sum(m for m, i in zip(lens, ids) if i == 1)
            assert torch.equal(got[torch.from_numpy(whole).to(cuda)], ref[torch.from_numpy(whole).to(cuda)])
            np.testing.assert_array_equal(got.double().cpu().numpy()[~whole], want[~whole])


@pytest.mark.parametrize("m", [9, 600])
def test_inner_sums_past_the_parts_range(mpq, cuda, m):
    """One infinity in `down`, and sums beside it that 16 bits do not hold: the row's results are infinities by the signs of up, not NaN."""
    c = Case(mpq, cuda, [m], [0], 1300, 64, 16, "f16")
    c.factor = c.factor * 1e7
    c.down[0, 3, 5] = math.inf
    c.low = mpq.adapters(c.down.to(cuda), c.up.to(cuda), c.factor.to(cuda))
    with np.errstate(invalid="ignore"):
        want = sum(c.sums()[:2])
    assert np.isinf(want).all()
    np.testing.assert_array_equal(c.run().double().cpu().numpy(), want)
