"""Level bytes with one range per row: the norm with the residual's addition and the row encoder,
against 64-bit arithmetic and against the quantizer's own 32-bit rule."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (1, 4096), (3, 7), (5, 64), (2, 255), (4, 1000), (7, 4104), (3, 9216), (2, 16384), (2, 16391), (1, 40000), (300, 130)]


def rand(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g) * scale


def row_range_exact(x, hrelu=False):
    x = np.where(np.isnan(x), 0, x)
    return (np.maximum(x, 0) if hrelu else np.abs(x)).max(1).astype(np.float32)


def row_levels(x, s, bits, hrelu=False):
    """The quantizer's rule in 32 bits (two rounded products, floor), as numpy computes it."""
    H, half_L = 1 << (bits - 1), np.float32(((1 << bits) - 1) / 2)
    inv = np.zeros_like(s)
    ok = np.isfinite(s) & (s > 0)
    inv[ok] = np.float32(1) / s[ok]
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x * inv[:, None]) * half_L
    y = np.where(np.isnan(y), np.float32(0), y)
    if hrelu:
        y = np.maximum(y, 0)
    return np.floor(np.clip(y, -H, H - 0.5)).astype(np.int64) + H


def check_held(lv, rows, k, bits):
    """Padding, level sums and the width of the levels; returns the levels as int64."""
    held = lv.bytes.cpu().numpy().astype(np.int64)
    assert held.shape == (rows, -(-k // 16) * 16)
    assert not held[:, k:].any()
    assert held.max(initial=0) < (1 << bits)
    assert np.array_equal(held.sum(1), lv.sums.cpu().numpy())
    return held[:, :k]


@pytest.mark.parametrize("rows,k", SHAPES)
@pytest.mark.parametrize("name", list(TYPES))
def test_encode_levels_follows_the_quantizer_exactly(mpq, cuda, rows, k, name):
    for bits, act in ((8, mpq.ACT_HTANH), (4, mpq.ACT_HTANH), (1, mpq.ACT_HTANH), (5, mpq.ACT_HRELU)):
        x = rand((rows, k), rows * 31 + k + bits).to(TYPES[name])
        values = torch.empty((rows, k), dtype=torch.float32, device=cuda)
        lv = mpq.encode_levels(x.to(cuda), bits, act, values=values)
        xf = x.float().numpy()
        s = row_range_exact(xf, act == mpq.ACT_HRELU)
        assert np.array_equal(lv.scale.cpu().numpy(), s)
        u = check_held(lv, rows, k, bits)
        assert np.array_equal(u, row_levels(xf, s, bits, act == mpq.ACT_HRELU))
        L = (1 << bits) - 1
        assert np.array_equal(values.cpu().numpy(), (2 * u - L).astype(np.float32) * (s / np.float32(L))[:, None])


def test_levels_agree_with_the_bit_planes(mpq, cuda):
    """The same quantizer as mpq_encode with one range per row: plane p holds bit p of the level byte."""
    x = rand((9, 333), 5).to(cuda)
    for bits in (2, 8):
        lv = mpq.encode_levels(x, bits)
        scale, planes = mpq.encode_ranged(x, bits)
        assert torch.equal(scale, lv.scale)
        words = planes.cpu().numpy().view(np.uint32)
        got = np.zeros((9, words.shape[2] * 32), dtype=np.int64)
        for p in range(bits):
            got += (((words[p][:, :, None] >> np.arange(32, dtype=np.uint32)) & 1).reshape(9, -1)).astype(np.int64) << p
        assert np.array_equal(got[:, :333], lv.bytes.cpu().numpy()[:, :333])


def test_encode_levels_special_rows(mpq, cuda):
    x = rand((6, 48), 3)
    x[0] = 0                                   # no range: every element lands on the level above zero
    x[1, 7] = float("nan")                     # a NaN takes no part in the range and lands there too
    x[2] = float("nan")
    x[3, 0] = float("inf")
    x[4] = 1e-42                               # subnormal
    x[5] = -x[5].abs()
    lv = mpq.encode_levels(x.to(cuda), 8)
    xf = x.numpy()
    s = row_range_exact(xf)
    assert np.array_equal(lv.scale.cpu().numpy(), s)
    u = check_held(lv, 6, 48, 8)
    assert (u[0] == 128).all() and u[1, 7] == 128 and (u[2] == 128).all() and (u[3] == 128).all()
    ok = [1, 5]
    assert np.array_equal(u[ok], row_levels(xf, s, 8)[ok])
    hr = mpq.encode_levels(x[5:].to(cuda), 8, mpq.ACT_HRELU)
    assert float(hr.scale[0]) == 0.0 and (hr.bytes[0, :48] == 128).all()


def norm_reference(x, r, gain, eps, bits):
    h = x.double() + (r.double() if r is not None else 0)
    y = h / torch.sqrt((h * h).mean(1, keepdim=True) + eps)
    if gain is not None:
        y = y * gain.double()
    s = y.abs().amax(1)
    return h, y.numpy(), s.numpy()


@pytest.mark.parametrize("rows,k", SHAPES)
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("with_res", [False, True])
def test_norm_against_64_bits(mpq, cuda, rows, k, name, with_res):
    """Relative error of y and its range: the sum of squares of k terms is at most 64 roundings deep per lane plus
    the tree (2^-24 each, half of it after the root), four more for quotient, root and products: under 5e-6.  A
    level may then differ (by one) only where (L/2) y / s lies within L/2 * 1e-5 of a boundary."""
    bits = 8
    x = rand((rows, k), rows + k).to(TYPES[name])
    r = rand((rows, k), rows + k + 1, 2.0).to(TYPES[name]) if with_res else None
    gain = 1 + 0.3 * rand((k,), 9)
    eps = 1e-5
    vt = torch.float16 if name == "f16" else torch.bfloat16
    values = torch.empty((rows, k), dtype=vt, device=cuda)
    ho = torch.empty((rows, k), dtype=TYPES[name], device=cuda)
    lv = mpq.rmsnorm_levels(x.to(cuda), gain.to(cuda), eps, bits, residual=None if r is None else r.to(cuda), residual_out=ho, values=values)
    h, y, s = norm_reference(x, r, gain, eps, bits)
    want_h = x.float() + r.float() if with_res else x.float()
    assert torch.equal(ho.cpu(), want_h.to(TYPES[name]))
    got_s = lv.scale.cpu().numpy()
    assert np.all(np.abs(got_s - s) <= 5e-6 * s)
    u = check_held(lv, rows, k, bits)
    t = 127.5 * y / s[:, None]
    want = np.floor(np.clip(t, -128, 127.5)).astype(np.int64) + 128
    off = u != want
    assert np.all(np.abs(u - want)[off] == 1)
    assert np.all(np.abs(t - np.round(t))[off] < 127.5e-5)
    back = (2 * u - 255).astype(np.float32) * (got_s / np.float32(255))[:, None]
    assert torch.equal(values.cpu(), torch.from_numpy(back).to(vt))


@pytest.mark.parametrize("bits", range(1, 9))
def test_norm_of_every_width_without_gain(mpq, cuda, bits):
    x = rand((4, 200), bits)
    lv = mpq.rmsnorm_levels(x.to(cuda), None, 0.0, bits)
    _, y, s = norm_reference(x, None, None, 0.0, bits)
    u, H, half_L = check_held(lv, 4, 200, bits), 1 << (bits - 1), ((1 << bits) - 1) / 2
    t = half_L * y / s[:, None]
    want = np.floor(np.clip(t, -H, H - 0.5)).astype(np.int64) + H
    assert np.all((u == want) | ((np.abs(u - want) == 1) & (np.abs(t - np.round(t)) < half_L * 1e-5)))


def test_norm_in_place_and_with_strides(mpq, cuda):
    """residual_out may be x or the residual; rows may lie apart and start anywhere."""
    wide = rand((6, 3, 515), 1).to(torch.bfloat16).to(cuda)
    for view in (wide[:, 0, :512], wide[:, 1, 1:513], wide[:, 2, 3:]):
        x, r = view.contiguous(), rand(view.shape, 2).to(torch.bfloat16).to(cuda)
        ref = mpq.rmsnorm_levels(x, None, 1e-6, 8, residual=r, residual_out=(h := torch.empty_like(x)))
        strided = mpq.rmsnorm_levels(view, None, 1e-6, 8, residual=r)
        assert torch.equal(ref.bytes, strided.bytes) and torch.equal(ref.scale, strided.scale)
        for target in ("x", "r"):
            xc, rc = x.clone(), r.clone()
            t = xc if target == "x" else rc
            got = mpq.rmsnorm_levels(xc, None, 1e-6, 8, residual=rc, residual_out=t)
            assert torch.equal(t, h) and torch.equal(got.bytes, ref.bytes)
    long = rand((2, 40001), 4).to(cuda)        # rows that are read twice
    r = rand((2, 40001), 5).to(cuda)
    ref = mpq.rmsnorm_levels(long, None, 1e-6, 8, residual=r, residual_out=(h := torch.empty_like(long)))
    got = mpq.rmsnorm_levels(long, None, 1e-6, 8, residual=r, residual_out=long)
    assert torch.equal(long, h) and torch.equal(got.bytes, ref.bytes)


def test_norm_special_rows(mpq, cuda):
    x = rand((4, 64), 8)
    x[0] = 0
    x[1, 3] = float("nan")
    x[2, 3] = float("inf")
    values = torch.empty((4, 64), dtype=torch.float32, device=cuda)
    lv = mpq.rmsnorm_levels(x.to(cuda), None, 1e-6, 8, values=values)
    s = lv.scale.cpu()
    assert s[0] == 0 and torch.isnan(s[1]) and torch.isnan(s[2]) and torch.isfinite(s[3])
    v = values.cpu()
    assert (v[0] == 0).all() and torch.isnan(v[1]).all() and torch.isnan(v[2]).all() and torch.isfinite(v[3]).all()


def test_no_rows_is_a_call_that_does_nothing(mpq, cuda):
    x = torch.empty((0, 64), device=cuda)
    assert mpq.rmsnorm_levels(x, None, 1e-6, 8).bytes.shape == (0, 64)
    assert mpq.encode_levels(x, 8).bytes.shape == (0, 64)


def test_on_another_stream(mpq, cuda):
    x = rand((64, 1024), 6).to(cuda)
    ref = mpq.rmsnorm_levels(x, None, 1e-6, 8)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        got = mpq.rmsnorm_levels(x, None, 1e-6, 8)
    st.synchronize()
    assert torch.equal(got.bytes, ref.bytes)
