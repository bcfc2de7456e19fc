"""Rows of the norm whose values are not ordinary: infinities and NaNs behind any gain."""
import pytest
import torch

pytestmark = pytest.mark.gpu

SIZES = [16, 64, 333, 4096, 9000, 40000]             # one warp, odd sizes, several vectors a thread, rows that are read twice


@pytest.mark.parametrize("k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_row_with_a_nan_or_an_infinity_gets_a_nan_range_whatever_the_gain(mpq, cuda, k, dtype):
    x = torch.randn((6, k), generator=torch.Generator().manual_seed(k))
    for row, value in ((1, float("inf")), (2, float("-inf")), (3, float("nan"))):
        x[row, k // 2] = value
    residual = torch.zeros((6, k))
    residual[4, 3] = float("inf")
    for g in (None, 0.0, 0.5, -2.0):
        gain = None
        if g is not None:
            gain = torch.ones(k)
            gain[k // 2] = gain[3] = g
        values = torch.empty((6, k), device=cuda)
        lv = mpq.rmsnorm_levels(x.to(dtype).to(cuda), None if gain is None else gain.to(cuda), 1e-6, 8,
                                residual=residual.to(dtype).to(cuda), values=values)
        assert torch.isnan(lv.scale[1:5]).all() and torch.isnan(values[1:5]).all()
        assert torch.isfinite(lv.scale[[0, 5]]).all() and torch.isfinite(values[[0, 5]]).all()
    gain = torch.ones(k)
    gain[1] = float("nan")                             # a NaN of the gain is one of every row
    assert torch.isnan(mpq.rmsnorm_levels(x.to(dtype).to(cuda), gain.to(cuda), 1e-6, 8).scale).all()
