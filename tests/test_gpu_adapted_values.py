"""Product of level bytes with adapters: infinities in them, and what 16-bit parts keep of the inner sums, and more
tiles than every pair of CTAs has accumulators."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_adapted import Case
from tests.test_gpu_linear_levels import TYPES, UNIT, activate

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


def check(c, act, out, bias=False, residual=False):
    """As Case.check, with what z loses in 16-bit parts: two bfloat16 parts leave (2^-8)^2 of each z at most, and so 2^-16 of the sizes
    that are added up; two float16 parts (2^-11)^2; an fp32 result has all of it.  Through the activation (slope at most 1.13)."""
    g = torch.Generator().manual_seed(9)
    b = torch.randn((c.n,), generator=g) if bias else None
    r = torch.randn((c.m, c.n), generator=g).to(TYPES[out]) if residual else None
    got = c.run(bias=None if b is None else b.to(c.cuda), act=act, residual=None if r is None else r.to(c.cuda), dtype=TYPES[out])
    f, delta, size = c.sums()
    whole = np.abs(f) + np.abs(delta)
    f = f + delta
    if bias:
        f, whole = f + b.double().numpy(), whole + np.abs(b.double().numpy())
    ref = activate(f, act) + (r.double().numpy() if residual else 0.0)
    lost = 2.0 ** -22 if c.down.dtype is torch.float16 else 0.0 if out == "f32" else 2.0 ** -16
    terms = 4 + math.sqrt(c.k + 128) / 4
    tol = UNIT[out] * np.abs(ref) + 16 * 2.0 ** -24 * (whole + np.abs(ref)) + 1.2 * (terms * 2.0 ** -24 + lost) * size + (2.0 ** -25 if out == "f16" else 0)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert got.dtype == TYPES[out] and np.all(err <= tol), (err - tol).max()


@pytest.mark.parametrize("lens,n", [([9], 300), ([600], 1601), ([300, 17, 283], 1601)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_what_z_keeps(mpq, cuda, lens, n, dtype):
    """Adapters whose terms cancel, beside a product of next to nothing: results of all types show no more than the parts of z lose."""
    c = Case(mpq, cuda, lens, [2, 0, 1][:len(lens)], n, 320, 64, dtype, seed=5)
    c.up[:, :, 32:] = -c.up[:, :, :32]
    c.down[:, 32:] = (c.down[:, :32].float() * (1 + 2.0 ** -6)).to(c.down.dtype)
    c.low = mpq.adapters(c.down.to(cuda), c.up.to(cuda), c.factor.to(cuda))
    c.w.scale.mul_(1e-4)
    c.sw = c.w.scale.double().cpu().numpy() / 255
    for out in ("f32", "f16", "bf16"):
        check(c, "none", out)


# pairs of CTAs have some three tiles of 256 x 128 and more each, so that both accumulators, and what adapters add beside them, are used
# again: tiles of one adapter, of several and of none one after the other
@pytest.mark.parametrize("out", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens,ids,n,rank", [([1300, 1, 1299], [1, -1, 0], 4000, 128), ([1300, 1, 1299], [1, -1, 0], 9000, 16), ([2600], [2], 4001, 64),
                                             ([256, 3, 509, 300, 700, 832], [0, 1, 2, -1, 3, 1], 5000, 16), ([100] * 26, [i % 5 - 1 for i in range(26)], 3900, 32),
                                             ([512, 512, 512, 512, 512, 40], [0, -1, 1, -1, 2, 3], 4200, 80)])
def test_more_tiles_than_accumulators(mpq, cuda, lens, ids, n, rank, dtype, out):
    assert -(-sum(lens) // 256) * -(-n // 128) > 3 * 74
    c = Case(mpq, cuda, lens, ids, n, 64, rank, dtype, seed=n)
    check(c, "none", out)
    check(c, "silu", out, True, True)
