"""What the decoder block's operators refuse, on a machine without a GPU: every error that the host can see comes back
as a status before anything is launched, and the binding refuses tensors that do not fit."""
import ctypes

import pytest
import torch

OK, NULL_, SHAPE, UNSUP, OVER, ALIGN, WORKSPACE = 0, 1, 2, 3, 4, 5, 7
N = None


@pytest.fixture(scope="module")
def mem():
    buf = (ctypes.c_uint32 * 64)()
    at = (ctypes.cast(buf, ctypes.c_void_p).value + 15) // 16 * 16
    return buf, ctypes.c_void_p(at), ctypes.c_void_p(at + 4), ctypes.c_void_p(at + 1)


def test_level_row_bytes(mpq):
    assert [mpq.level_row_bytes(k) for k in (1, 16, 17, 4096, 4100)] == [16, 16, 32, 4096, 4112]
    assert mpq.level_row_bytes(0) == 0 and mpq.level_row_bytes(-3) == 0


def test_norm_and_row_encoder(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def norm(x=p, ldx=64, res=N, ldr=0, dtype=0, gain=N, eps=1e-6, rows=4, k=64, bits=8, ho=N, ldo=0, lv=p, s=p, sums=p, v=N, vt=0, ldv=0):
        return L.mpq_rmsnorm_levels(x, ldx, res, ldr, dtype, gain, eps, rows, k, bits, ho, ldo, lv, s, sums, v, vt, ldv, N)
    assert norm(x=N) == NULL_ and norm(lv=N) == NULL_ and norm(s=N) == NULL_ and norm(sums=N) == NULL_
    assert norm(rows=-1) == SHAPE and norm(k=0) == SHAPE and norm(k=1 << 23) == SHAPE
    assert norm(ldx=63) == SHAPE and norm(res=p, ldr=63) == SHAPE and norm(ho=p, ldo=63) == SHAPE and norm(v=p, ldv=63) == SHAPE
    assert norm(dtype=3) == UNSUP and norm(dtype=-1) == UNSUP and norm(v=p, ldv=64, vt=9) == UNSUP
    assert norm(bits=0) == UNSUP and norm(bits=9) == UNSUP and norm(eps=-1.0) == UNSUP and norm(eps=float("nan")) == UNSUP
    assert norm(lv=odd) == ALIGN and norm(x=byte) == ALIGN and norm(gain=byte) == ALIGN and norm(s=byte) == ALIGN
    assert norm(rows=0, x=N, lv=N, s=N, sums=N) == OK

    def enc(x=p, ldx=64, dtype=0, rows=4, k=64, act=0, bits=8, lv=p):
        return L.mpq_encode_levels(x, ldx, dtype, rows, k, act, bits, lv, p, p, N, 0, 0, N)
    assert enc(x=N) == NULL_ and enc(ldx=10) == SHAPE and enc(act=2) == UNSUP and enc(bits=12) == UNSUP and enc(lv=odd) == ALIGN
    assert enc(rows=0) == OK


def test_linear(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def lin(a=p, sa=p, ua=p, ab=8, w=p, sw=p, uw=p, wb=8, m=4, n=8, k=64, bias=N, glue=0, res=N, ldr=0, out=p, dtype=0, ldo=8):
        return L.mpq_linear_levels(a, sa, ua, ab, w, sw, uw, wb, m, n, k, bias, glue, res, ldr, out, dtype, ldo, N)
    for name in ("a", "sa", "ua", "w", "sw", "uw", "out"):
        assert lin(**{name: N}) == NULL_
    assert lin(m=-1) == SHAPE and lin(n=0) == SHAPE and lin(k=0) == SHAPE and lin(ldo=7) == SHAPE and lin(res=p, ldr=7) == SHAPE
    assert lin(ab=0) == UNSUP and lin(wb=9) == UNSUP and lin(dtype=3) == UNSUP and lin(glue=5) == UNSUP and lin(glue=-1) == UNSUP
    assert lin(k=33026) == OVER and lin(ab=1, wb=1, k=2 ** 31) == OVER
    assert lin(a=odd) == ALIGN and lin(w=odd) == ALIGN and lin(out=byte) == ALIGN and lin(bias=byte) == ALIGN
    assert lin(m=0, a=N, out=N) == OK


def test_cache(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def write(k=p, kt=64, kh=64, v=p, vt=64, vh=64, dtype=0, slots=p, tokens=2, heads=1, dim=64, bits=8, kl=p, ks=p, vl=p, vs=p, pages=2, page=4):
        return L.mpq_cache_write(k, kt, kh, v, vt, vh, dtype, slots, tokens, heads, dim, bits, kl, ks, vl, vs, pages, page, N)

    def read(k=p, kt=64, kh=64, v=p, vt=64, vh=64, dtype=0, slots=p, tokens=2, heads=1, dim=64, bits=8, kl=p, ks=p, vl=p, vs=p, pages=2, page=4):
        return L.mpq_cache_read(kl, ks, vl, vs, pages, page, slots, tokens, heads, dim, bits, k, kt, kh, v, vt, vh, dtype, N)
    for f in (write, read):
        for name in ("k", "v", "slots", "kl", "ks", "vl", "vs"):
            assert f(**{name: N}) == NULL_
        assert f(tokens=-1) == SHAPE and f(heads=0) == SHAPE and f(pages=0) == SHAPE and f(page=0) == SHAPE
        assert f(dtype=3) == UNSUP and f(bits=5) == UNSUP and f(dim=48) == UNSUP and f(dim=0) == UNSUP and f(dim=288) == UNSUP
        assert f(kl=odd) == ALIGN and f(k=byte) == ALIGN and f(vs=byte) == ALIGN and f(slots=odd) == ALIGN
        assert f(tokens=0, k=N, v=N) == OK
    assert read(kt=63) == SHAPE and read(heads=2, vh=63, kt=128, vt=128) == SHAPE


def test_attention(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def attn(q=p, qt=256, qh=64, dtype=1, starts=p, lens=p, table=p, stride=4, tokens=2, batch=1, heads=4, kv=2, dim=64, mq=2, mk=64,
             kl=p, ks=p, vl=p, vs=p, bits=8, pages=4, page=16, causal=1, window=0, scale=0.125, out=p, ot=256, oh=64, lse=N, ws=N, wsb=0):
        return L.mpq_cache_attention(q, qt, qh, dtype, starts, lens, table, stride, tokens, batch, heads, kv, dim, mq, mk, kl, ks, vl, vs,
                                     bits, pages, page, causal, window, scale, out, ot, oh, lse, ws, wsb, N)
    for name in ("q", "starts", "lens", "table", "kl", "ks", "vl", "vs", "out"):
        assert attn(**{name: N}) == NULL_
    assert attn(tokens=-1) == SHAPE and attn(batch=0) == SHAPE and attn(heads=3) == SHAPE and attn(kv=0) == SHAPE and attn(pages=0) == SHAPE
    assert attn(stride=0) == SHAPE and attn(page=0) == SHAPE and attn(window=-1) == SHAPE and attn(ot=63) == SHAPE and attn(oh=63) == SHAPE
    assert attn(mq=-1) == SHAPE and attn(mk=-1) == SHAPE
    assert attn(dtype=0) == UNSUP and attn(bits=2) == UNSUP and attn(dim=96) == UNSUP
    assert attn(scale=float("nan")) == UNSUP and attn(scale=float("inf")) == UNSUP
    assert attn(kl=odd) == ALIGN and attn(q=byte) == ALIGN and attn(lse=byte) == ALIGN and attn(table=byte) == ALIGN
    assert attn(tokens=0, q=N, out=N) == OK
    need = mpq.cache_attention_workspace(2, 1, 4, 2, 64, 1, 100000)
    assert need > 0
    assert attn(mq=1, mk=100000) == NULL_ and attn(mq=1, mk=100000, ws=p, wsb=need - 1) == WORKSPACE and attn(mq=1, mk=100000, ws=odd, wsb=need) == ALIGN
    assert mpq.cache_attention_workspace(2, 1, 4, 3, 64, 1, 100) == 0 and mpq.cache_attention_workspace(0, 1, 4, 2, 64, 1, 100) == 0


def test_binding_refusals(mpq):
    x = torch.zeros((4, 64))
    with pytest.raises(ValueError):
        mpq.rmsnorm_levels(x, None, 1e-6)                     # a host tensor
    with pytest.raises(ValueError):
        mpq.encode_levels(x)
    lv = mpq.Levels(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros(4), torch.zeros(4, dtype=torch.int32), 8, 64)
    with pytest.raises(ValueError):
        mpq.linear_levels(lv, lv, act="swish")
    with pytest.raises(ValueError):
        mpq.linear_levels(lv, lv._replace(k=63))
    cache = mpq.level_cache(2, 1, 4, 64, 8, "cpu")
    with pytest.raises(ValueError):
        mpq.cache_write(cache, torch.zeros((2, 1, 64)), torch.zeros((2, 1, 64)), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        mpq.cache_attention(torch.zeros((2, 1, 64)), cache, torch.zeros(2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32),
                            torch.zeros((1, 2), dtype=torch.int32), 2, 4)
