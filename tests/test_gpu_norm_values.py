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


@pytest.mark.parametrize("k", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("with_residual", [False, True])
def test_finite_rows_of_any_size_keep_their_range(mpq, cuda, k, dtype, with_residual):
    """Rows whose squares, or the sum of whose squares, leave the 32-bit range.  Tolerance as in the norm's 64-bit test,
    5e-6 of the range (the sum at most 64 roundings of 2^-24 deep, root, quotients, products), and 2^-21 more for a factor
    that is subnormal at the very largest elements; levels differ by one, near a boundary, at most."""
    g = torch.Generator().manual_seed(k)
    x = torch.randn((8, k), generator=g)
    for row, power in enumerate((44, 50, 62, 64, 80, 120)):
        x[row] = (x[row] * 2.0 ** power).clamp(-1e38, 1e38)
    x[6, k // 3] = 2e38                                # one element has nearly all of the row
    x[7, :] = 1.0
    x[7, k - 1] = -2.0 ** 70
    x = x.to(dtype)
    r = (x.float() * torch.rand((8, k), generator=g) * 0.5).to(dtype) if with_residual else None
    gain = 0.25 + 0.5 * torch.rand((k,), generator=g)
    gain[k // 2] = 0.0
    h = x.double() + (r.double() if with_residual else 0.0)
    for eps in (0.0, 1e-6, 1e30):
        for in_place in (False, True):
            rel = 5e-6 + 2.0 ** -21
            values = torch.empty((8, k), device=cuda)
            xd = x.to(cuda)
            lv = mpq.rmsnorm_levels(xd, gain.to(cuda), eps, 8, residual=None if r is None else r.to(cuda),
                                    residual_out=xd if in_place else None, values=values)
            if in_place:
                assert torch.equal(xd.cpu(), (x.float() + (r.float() if with_residual else 0.0)).to(dtype))
            y = h / torch.sqrt((h * h).mean(1, keepdim=True) + float(torch.tensor(eps, dtype=torch.float32))) * gain.double()
            s = y.abs().amax(1)
            got = lv.scale.double().cpu()
            assert ((got - s).abs() <= rel * s).all(), (got / s - 1)
            t = 127.5 * y / s[:, None]
            want = (torch.floor(t.clamp(-128, 127.5)) + 128).long()
            u = lv.bytes[:, :k].long().cpu()
            off = u != want
            assert ((u - want).abs()[off] <= 1).all() and ((t - t.round()).abs()[off] < 127.5 * 2 * rel).all()
            back = (2 * u - 255).float() * (lv.scale.cpu() / 255)[:, None]
            assert torch.equal(values.cpu(), back)
