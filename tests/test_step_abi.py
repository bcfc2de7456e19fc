"""What the operators around a server's step refuse, on a machine without a GPU: every error that the host can see comes back
as a status before anything is launched."""
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


def test_pages(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def extend(table=p, per=4, lens=p, sequences=3, free=p, pages=9, count=p, page=16, seqs=p, new=p, batch=2, tokens=5, slots=p, starts=p, kv=p,
               rows=p, missing=p):
        return L.mpq_pages_extend(table, per, lens, sequences, free, pages, count, page, seqs, new, batch, tokens, slots, starts, kv, rows, missing, N)

    def trim(table=p, per=4, lens=p, sequences=3, free=p, pages=9, count=p, page=16, seqs=p, keep=p, batch=2):
        return L.mpq_pages_trim(table, per, lens, sequences, free, pages, count, page, seqs, keep, batch, N)
    for name in ("table", "lens", "free", "count", "new", "slots", "starts", "kv", "rows", "missing"):
        assert extend(**{name: N}) == NULL_, name
        assert extend(**{name: byte}) == ALIGN, name
    assert extend(slots=odd) == ALIGN and extend(seqs=byte) == ALIGN
    for name in ("table", "lens", "free", "count", "keep"):
        assert trim(**{name: N}) == NULL_, name
        assert trim(**{name: byte}) == ALIGN, name
    for call in (extend, trim):
        for bad in (dict(per=0), dict(sequences=0), dict(pages=0), dict(pages=2 ** 31), dict(page=0), dict(page=-4), dict(batch=-1),
                    dict(per=2 ** 27), dict(seqs=N, batch=4)):
            assert call(**bad) == SHAPE, bad
        assert call(batch=8193) == UNSUP
    assert extend(tokens=-1) == SHAPE and extend(tokens=2 ** 31) == SHAPE


def test_linear_adapted(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def lin(a=p, sa=p, ua=p, ab=8, w=p, sw=p, uw=p, wb=8, m=4, n=8, k=64, down=p, up=p, at=1, factor=N, adapters=2, rank=16, starts=p, ids=p, batch=3,
            bias=N, glue=0, res=N, ldr=0, out=p, dtype=0, ldo=8, ws=p, wb_=1 << 20):
        return L.mpq_linear_adapted(a, sa, ua, ab, w, sw, uw, wb, m, n, k, down, up, at, factor, adapters, rank, starts, ids, batch, bias, glue, res, ldr,
                                    out, dtype, ldo, ws, wb_, N)
    for name in ("a", "sa", "ua", "w", "sw", "uw", "out", "down", "up", "starts", "ids", "ws"):
        assert lin(**{name: N}) == NULL_, name
    assert lin(m=-1) == SHAPE and lin(n=0) == SHAPE and lin(k=0) == SHAPE and lin(ldo=7) == SHAPE and lin(res=p, ldr=7) == SHAPE
    assert lin(adapters=0) == SHAPE and lin(rank=0) == SHAPE and lin(rank=-16) == SHAPE and lin(batch=-1) == SHAPE
    assert lin(adapters=1 << 29) == SHAPE and lin(m=1 << 30, ldo=8) == SHAPE
    assert lin(ab=0) == UNSUP and lin(wb=9) == UNSUP and lin(dtype=3) == UNSUP and lin(glue=5) == UNSUP
    assert lin(at=0) == UNSUP and lin(at=3) == UNSUP and lin(rank=8) == UNSUP and lin(rank=24) == UNSUP and lin(rank=144) == UNSUP
    assert lin(k=33026) == OVER
    for name in ("a", "w", "down", "up", "ws"):
        assert lin(**{name: odd}) == ALIGN, name
    for name in ("factor", "starts", "ids", "bias", "out"):
        assert lin(**{name: byte}) == ALIGN, name
    need = mpq.linear_adapted_workspace(4, 16)
    assert need > 0 and need % 16 == 0 and lin(wb_=need - 1) == WORKSPACE
    assert mpq.linear_adapted_workspace(0, 16) == 0 and mpq.linear_adapted_workspace(5, 0) == 0 and mpq.linear_adapted_workspace(1, 16) == (10 * 16 + 8 + 15) // 16 * 16
    assert lin(m=0, a=N, out=N, ws=N, wb_=0) == OK


def test_sample(mpq, mem):
    L, (_, p, odd, byte) = mpq.lib(), mem

    def draw(x=p, ld=64, dtype=0, rows=2, vocab=64, t=N, k=N, tp=N, mp=N, u=p, out=p, lp=N):
        return L.mpq_sample(x, ld, dtype, rows, vocab, t, k, tp, mp, u, out, lp, N)
    for name in ("x", "u", "out"):
        assert draw(**{name: N}) == NULL_, name
    assert draw(rows=-1) == SHAPE and draw(vocab=0) == SHAPE and draw(ld=63) == SHAPE and draw(rows=2 ** 31, ld=64) == SHAPE
    assert draw(dtype=3) == UNSUP and draw(dtype=-1) == UNSUP
    assert draw(vocab=393217, ld=393217) == UNSUP and draw(vocab=786433, ld=786433, dtype=2) == UNSUP
    for name in ("x", "t", "k", "tp", "mp", "u", "out", "lp"):
        assert draw(**{name: byte}) == ALIGN, name
    assert draw(out=odd) == ALIGN
    assert draw(rows=0, x=N, u=N, out=N) == OK


def test_adapters_are_laid_out(mpq):
    down, up = torch.randn((3, 5, 20)).half(), torch.randn((3, 7, 5)).half()
    low = mpq.adapters(down, up, torch.ones(3))
    assert low.down.shape == (3, 16, 32) and low.up.shape == (3, 7, 16) and low.k == 20
    assert torch.equal(low.down[:, :5, :20], down) and torch.equal(low.up[:, :, :5], up)
    assert not low.down[:, 5:].any() and not low.down[:, :, 20:].any() and not low.up[:, :, 5:].any()
    for bad in ((down, up[:2]), (down, up[:, :, :4]), (down, up.float()), (down, up, torch.ones(2))):
        with pytest.raises(ValueError):
            mpq.adapters(*bad)


def test_host_tensors_are_refused(mpq):
    state = mpq.page_state(2, 4, 8, 16, "cpu")
    ints = torch.zeros(2, dtype=torch.int32)
    assert state.free.tolist() == [7, 6, 5, 4, 3, 2, 1, 0] and state.count.tolist() == [8, 0]
    for call in (lambda: mpq.pages_extend(state, None, ints, 4), lambda: mpq.pages_trim(state, ints, ints), lambda: mpq.sample(torch.zeros((2, 9)), torch.zeros(2))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
