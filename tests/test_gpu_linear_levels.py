"""Product of level bytes with bias, activation and residual in its epilogue, against int64 products and
64-bit arithmetic."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}       # a rounding, relative (bf16: a whole unit's half is 2^-9)


def operand(mpq, cuda, rows, k, bits, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    u = torch.randint(0, 1 << bits, (rows, k), generator=g)
    held = torch.zeros((rows, -(-k // 16) * 16), dtype=torch.uint8)
    held[:, :k] = u.to(torch.uint8)
    scale = torch.rand((rows,), generator=g) * std + 0.01
    lv = mpq.Levels(held.to(cuda), scale.to(cuda), u.sum(1).to(torch.int32).to(cuda), bits, k)
    return lv, (2 * u - ((1 << bits) - 1)).numpy().astype(np.int64), scale.numpy().astype(np.float64) / ((1 << bits) - 1)


def activate(y, act):
    if act == "relu":
        return np.maximum(y, 0)
    if act == "gelu":
        return y * 0.5 * np.vectorize(math.erfc)(-y / math.sqrt(2))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + np.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3)))
    if act == "silu":
        return y / (1 + np.exp(-y))
    return y


def check(mpq, cuda, m, n, k, a_bits, w_bits, act, bias, residual, out_type, seed):
    a, qa, sa = operand(mpq, cuda, m, k, a_bits, seed)
    w, qw, sw = operand(mpq, cuda, n, k, w_bits, seed + 1, std=2.0 / math.sqrt(k))
    g = torch.Generator().manual_seed(seed + 2)
    b = torch.randn((n,), generator=g) if bias else None
    r = torch.randn((m, n), generator=g).to(TYPES[out_type]) if residual else None
    got = mpq.linear_levels(a, w, bias=None if b is None else b.to(cuda), act=act, residual=None if r is None else r.to(cuda), dtype=TYPES[out_type])
    acc = (qa.astype(np.float64) @ qw.T.astype(np.float64))                  # exact: below 2^53
    f = acc * (sa[:, None] * sw[None, :])
    size = np.abs(f)
    if bias:
        f = f + b.numpy().astype(np.float64)
        size = size + np.abs(b.numpy())
    y = activate(f, act)
    ref = y + r.double().numpy() if residual else y
    # float(acc), two range quotients and their product, the product, the bias: 6 roundings of 2^-24; the smooth
    # activations have slope at most 1.13 and an error of their own of 8 units of the argument's size; one last rounding
    tol = UNIT[out_type] * np.abs(ref) + 16 * 2.0 ** -24 * (size + np.abs(ref)) + (2.0 ** -25 if out_type == "f16" else 0)
    err = np.abs(got.double().cpu().numpy() - ref)
    assert got.dtype == TYPES[out_type] and got.shape == (m, n)
    assert np.all(err <= tol), (err - tol).max()


SIZES = [(1, 1, 1), (1, 64, 16), (2, 5, 33), (3, 130, 100), (8, 1000, 512), (9, 257, 4100), (16, 64, 128), (17, 100, 640), (33, 4096, 64),
         (64, 300, 1024), (65, 31, 31), (128, 256, 256), (129, 257, 272), (200, 1003, 777), (256, 512, 1040), (1000, 120, 48), (300, 77, 2050)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_sizes(mpq, cuda, m, n, k):
    check(mpq, cuda, m, n, k, 8, 8, "none", False, False, "f32", m + n + k)
    check(mpq, cuda, m, n, k, 8, 8, "silu", True, True, "bf16", m + n + k + 5)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("out_type", list(TYPES))
@pytest.mark.parametrize("m", [1, 20, 150])
def test_epilogues(mpq, cuda, act, out_type, m):
    for bias, residual in ((False, False), (True, False), (False, True), (True, True)):
        check(mpq, cuda, m, 200, 320, 8, 8, act, bias, residual, out_type, 77)


# more 128 x 64 tiles than multiprocessors: CTA pairs, with one tile each, with several, with rows and columns left over
MANY = [(513, 2177, 272), (777, 1601, 100), (2600, 1201, 200), (4097, 1001, 130), (1024, 2560, 512), (130, 9001, 48)]


@pytest.mark.parametrize("m,n,k", MANY)
@pytest.mark.parametrize("out_type", list(TYPES))
def test_many_tiles(mpq, cuda, m, n, k, out_type):
    check(mpq, cuda, m, n, k, 8, 8, "none", False, False, out_type, m + n + k)
    check(mpq, cuda, m, n, k, 8, 8, "silu", True, True, out_type, m + n + k + 5)
    check(mpq, cuda, m, n, k, 3, 5, "gelu", True, True, out_type, m + n + k + 6)


@pytest.mark.parametrize("a_bits,w_bits", [(1, 1), (8, 1), (2, 8), (4, 4), (5, 3)])
@pytest.mark.parametrize("m", [2, 40, 140])
def test_widths(mpq, cuda, a_bits, w_bits, m):
    check(mpq, cuda, m, 150, 500, a_bits, w_bits, "none", True, False, "f32", 3)


@pytest.mark.parametrize("m", [1, 7, 30, 130, 513])
def test_largest_sums_are_exact(mpq, cuda, m):
    """k at the edge of int32 with every level at its end: the sums reach +-(2^31 - 66,000)."""
    k, n = 33025, 5
    top = lambda rows, v: mpq.Levels(torch.nn.functional.pad(torch.full((rows, k), v, dtype=torch.uint8), (0, -k % 16)).to(cuda),      # noqa: E731
                                     torch.full((rows,), 255.0, device=cuda), torch.full((rows,), k * v, dtype=torch.int32, device=cuda), 8, k)
    for va, vw, sign in ((255, 255, 1), (255, 0, -1), (0, 0, 1)):
        got = mpq.linear_levels(top(m, va), top(n, vw))
        assert (got.cpu() == float(np.float32(sign * k * 255 * 255))).all()


def test_agrees_with_the_bit_plane_product(mpq, cuda):
    g = torch.Generator().manual_seed(1)
    x, w = torch.randn((12, 300), generator=g).to(cuda), torch.randn((40, 300), generator=g).to(cuda)
    a, b = mpq.encode_levels(x[:1].expand(12, 300).contiguous(), 3), mpq.encode_levels(w, 2)
    got = mpq.linear_levels(a, b)
    s_a = a.scale[:1].contiguous()
    ap = mpq.encode(x[:1].expand(12, 300).contiguous(), s_a, 3)
    ws, wp = mpq.encode_ranged(w, 2)
    ci = torch.empty((12, 40), dtype=torch.int32, device=cuda)
    cf = torch.empty((12, 40), dtype=torch.float32, device=cuda)
    mpq.gemm(ap, 3, wp, 2, 12, 40, 300, ci, cf, s_a, ws, mpq.SCALE_PER_ROW)
    assert torch.equal(got, cf)


def test_output_over_its_residual_and_strided(mpq, cuda):
    a, _, _ = operand(mpq, cuda, 37, 96, 8, 1)
    w, _, _ = operand(mpq, cuda, 50, 96, 8, 2)
    for dt in TYPES.values():
        wide = torch.randn((37, 120), device=cuda).to(dt)
        for at in (0, 3, 8):
            view = wide[:, at:at + 50]
            ref = mpq.linear_levels(a, w, residual=view.contiguous(), dtype=dt)
            buf = wide.clone()
            got = mpq.linear_levels(a, w, residual=buf[:, at:at + 50], out=buf[:, at:at + 50])
            assert torch.equal(got, ref)
            assert torch.equal(buf[:, :at], wide[:, :at]) and torch.equal(buf[:, at + 50:], wide[:, at + 50:])


def test_non_finite_ranges_stay_in_their_row_and_column(mpq, cuda):
    a, _, _ = operand(mpq, cuda, 20, 64, 8, 4)
    w, _, _ = operand(mpq, cuda, 30, 64, 8, 5)
    ref = mpq.linear_levels(a, w)
    a.scale[3] = float("nan")
    w.scale[7] = float("inf")
    got = mpq.linear_levels(a, w)
    assert torch.isnan(got[3]).all() and not torch.isfinite(got[:, 7]).any()
    keep_r, keep_c = [i for i in range(20) if i != 3], [i for i in range(30) if i != 7]
    assert torch.equal(got[keep_r][:, keep_c], ref[keep_r][:, keep_c])


def test_no_rows_and_another_stream(mpq, cuda):
    a, _, _ = operand(mpq, cuda, 140, 256, 8, 4)
    w, _, _ = operand(mpq, cuda, 300, 256, 8, 5)
    empty = mpq.Levels(a.bytes[:0], a.scale[:0], a.sums[:0], 8, 256)
    assert mpq.linear_levels(empty, w).shape == (0, 300)
    for rows in (1, 16, 140):
        part = mpq.Levels(a.bytes[:rows], a.scale[:rows], a.sums[:rows], 8, 256)
        ref = mpq.linear_levels(part, w)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            got = mpq.linear_levels(part, w)
        st.synchronize()
        assert torch.equal(got, ref)


def test_no_wait_ran_out(mpq, cuda):
    """After every product above: no CTA gave up waiting for its copies or its partner."""
    assert mpq.wait_failures() == 0
