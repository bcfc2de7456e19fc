"""Tensors that the binding of the calls around a step refuses because they are elsewhere."""
import pytest
import torch

from tests.test_gpu_block_binding import Elsewhere

pytestmark = pytest.mark.gpu


def every_call(mpq, cuda):
    """name -> (call, its tensors)"""
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=cuda)                          # noqa: E731
    a, w = (mpq.encode_levels(torch.randn((rows, 64), device=cuda)) for rows in (6, 8))
    low = mpq.adapters(torch.randn((2, 16, 64), device=cuda).half(), torch.randn((2, 8, 16), device=cuda).half(), torch.ones(2, device=cuda))
    held = lambda lv, *t: mpq.Levels(*t, lv.bits, lv.k)                                        # noqa: E731
    state = mpq.page_state(3, 4, 12, 16, cuda)
    one = torch.full((4,), 0.5, device=cuda)
    return {
        "extend": (lambda t, n, f, c, q, m, s, st, kv, b, miss: mpq.pages_extend(mpq.PageState(t, n, f, c, 16), q, m, 4, mpq.PagePlan(s, st, kv, b, miss)),
                   [*state[:4], ints(0, 1), ints(1, 1), *mpq.pages_extend(state, ints(0, 1), ints(1, 1), 4)]),
        "trim": (lambda t, n, f, c, q, k: mpq.pages_trim(mpq.PageState(t, n, f, c, 16), q, k), [*state[:4], ints(0, 1), ints(0, 0)]),
        "adapted": (lambda ab, as_, au, wb, ws, wu, d, u, f, st, i, b, r, o, ws_: mpq.linear_adapted(
            held(a, ab, as_, au), held(w, wb, ws, wu), mpq.Adapters(d, u, f, 64), st, i, bias=b, residual=r, out=o, workspace=ws_),
            [*a[:3], *w[:3], *low[:3], ints(0, 4, 6), ints(0, 1), torch.zeros(8, device=cuda), torch.zeros((6, 8), device=cuda),
             torch.zeros((6, 8), device=cuda), torch.zeros(4096, device=cuda)]),
        "sample": (lambda x, u, t, k, p, m, o, lp: mpq.sample(x, u, t, k, p, m, o, lp),
                   [torch.randn((4, 50), device=cuda), one, one, ints(1, 2, 3, 4), one, one, torch.zeros(4, dtype=torch.int64, device=cuda), one.clone()]),
    }


def test_tensors_of_another_device_are_refused(mpq, cuda, monkeypatch):
    calls = every_call(mpq, cuda)
    for name, (call, tensors) in calls.items():
        call(*tensors)
        for i in range(len(tensors)):
            moved = list(tensors)
            moved[i] = moved[i].as_subclass(Elsewhere)
            with pytest.raises(ValueError):
                call(*moved)
                pytest.fail("%s took tensor %d from another device" % (name, i))
    monkeypatch.setattr(mpq, "_current_device", lambda: 1)
    for call, tensors in calls.values():
        with pytest.raises(ValueError, match="current device"):
            call(*tensors)


def test_calls_on_two_streams_at_once(mpq, cuda):
    """Each with its own state or workspace: none sees the other's."""
    g = torch.Generator().manual_seed(3)
    x = torch.randn((2, 40, 30000), generator=g).to(cuda)
    u, p = torch.rand((2, 40), generator=g).to(cuda), torch.full((40,), 0.9, device=cuda)
    a = [mpq.encode_levels(torch.randn((300, 640), generator=g).to(cuda)) for _ in range(2)]
    w = mpq.encode_levels(torch.randn((1700, 640), generator=g).to(cuda))
    low = mpq.adapters(torch.randn((3, 16, 640), generator=g).to(cuda).half(), torch.randn((3, 1700, 16), generator=g).to(cuda).half())
    starts, ids = torch.tensor([0, 100, 130, 300], dtype=torch.int32, device=cuda), torch.tensor([[2, 0, 1], [1, -1, 0]], dtype=torch.int32, device=cuda)
    work = lambda i: (mpq.sample(x[i], u[i], top_p=p), mpq.linear_adapted(a[i], w, low, starts, ids[i]))      # noqa: E731
    want = [work(0), work(1)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got.append((i, work(i)))
    torch.cuda.synchronize()
    for i, (tokens, out) in got:
        assert torch.equal(tokens, want[i][0]) and torch.equal(out, want[i][1])
