"""A server's step as a whole: pages and slots made on the device, adapters beside all products, tokens drawn -- against the
network in 64 bits, and captured once and replayed against the same step done with the host's bookkeeping."""
import pytest
import torch

from paper_1905_13389_b200 import decoder
from tests.test_gpu_decoder import reference, relative

pytestmark = pytest.mark.gpu

CONFIG = decoder.Config(layers=2, width=256, heads=8, kv_heads=2, dim=64, inner=768)


def ints(v, cuda):
    return torch.tensor(v, dtype=torch.int32, device=cuda)


def merged(weights, adapters, i):
    """The weights with adapter i added to them, in 64 bits."""
    out = []
    for w, low in zip(weights, adapters):
        w = {k: v.double() for k, v in w.items()}
        for name, a in low.items() if i >= 0 else ():
            w[name] = w[name] + a.scale[i].double() * (a.up[i].double() @ a.down[i, :, :a.k].double())
        out.append(w)
    return out


def test_against_64_bits(mpq, cuda):
    """Every sequence against the network with its own adapter merged into the weights.  The adapters are not quantized, so
    the tolerance is that of the network without them (test_gpu_decoder)."""
    weights, adapters = decoder.random_weights(CONFIG, cuda), decoder.random_adapters(CONFIG, 3, 24, cuda, 5)
    model, pages = decoder.EncodedDecoder(CONFIG, weights, 32, 16, adapters), decoder.DevicePages(32, 16, 4, 8, cuda)
    lens, ids = [70, 1, 33, 50], [2, 0, -1, 1]
    x = torch.randn((sum(lens), CONFIG.width), generator=torch.Generator().manual_seed(2)).to(cuda).to(torch.bfloat16)
    got = model.forward(x, pages.extend(None, ints(lens, cuda), sum(lens), 70, 70), ints(ids, cuda))
    pages.check()
    model.check()
    plain = model.forward(x, decoder.Pages(32, 16).extend(dict(enumerate(lens)), cuda))
    at = 0
    for n, i in zip(lens, ids):
        part = slice(at, at + n)
        ref = reference(CONFIG, merged(weights, adapters, i), x[part], [n])
        assert relative(got[part], ref) < 0.05
        if i >= 0:                                            # ... and the adapter is seen
            assert relative(plain[part], ref) > 0.08
        else:
            assert torch.equal(plain[part], got[part])
        at += n


def test_a_captured_step_serves_growing_sequences(mpq, cuda):
    """From lengths to tokens in one graph, three sequences and an entry of padding, replayed over a page's end; the same with the
    host's pages and eager calls gives the same tokens and hidden states, bit for bit."""
    weights, adapters = decoder.random_weights(CONFIG, cuda), decoder.random_adapters(CONFIG, 2, 16, cuda)
    g = torch.Generator().manual_seed(4)
    embedding = torch.randn((300, CONFIG.width), generator=g).to(cuda)
    words = mpq.encode_levels(embedding)
    lens, steps = [5, 14, 30], 9
    prompt = torch.randint(0, 300, (sum(lens),), generator=g).to(cuda)
    uniform = torch.rand((steps + 1, 4), generator=g).to(cuda)
    warm, top_k, top_p = torch.tensor([0.0, 0.7, 1.0, 1.0], device=cuda), ints([0, 40, 0, 0], cuda), torch.tensor([1.0, 1.0, 0.9, 1.0], device=cuda)
    ids = ints([1, -1, 0, 0], cuda)

    def draw(model, x, last, u):
        logits = mpq.linear_levels(mpq.rmsnorm_levels(x[last], None, CONFIG.eps), words)
        n = len(last)
        return mpq.sample(logits, u[:n], warm[:n], top_k[:n], top_p[:n])

    # with the host's pages
    model, pages = decoder.EncodedDecoder(CONFIG, weights, 16, 16, adapters), decoder.Pages(16, 16)
    batch = pages.extend(dict(enumerate(lens)), cuda)._replace(max_q=30, max_kv=64)
    x = model.forward(embedding[prompt].to(torch.bfloat16), batch, ids[:3])
    tokens = draw(model, x, batch.q_starts[1:].long() - 1, uniform[0])
    want, first = [tokens.tolist()], tokens.clone()
    for i in range(steps):
        batch = pages.extend({0: 1, 1: 1, 2: 1}, cuda)._replace(max_kv=64)
        x = model.forward(embedding[tokens].to(torch.bfloat16), batch, ids[:3])
        tokens = draw(model, x, torch.arange(3, device=cuda), uniform[i + 1])
        want.append(tokens.tolist())
    want_x = x

    # on the device, captured
    model, pages = decoder.EncodedDecoder(CONFIG, weights, 16, 16, adapters), decoder.DevicePages(16, 16, 6, 4, cuda)
    seqs = ints([4, 0, 2, -1], cuda)
    x = model.forward(embedding[prompt].to(torch.bfloat16), pages.extend(seqs, ints(lens + [0], cuda), len(prompt), 30, 64), ids)
    held = torch.zeros(4, dtype=torch.int64, device=cuda)
    held[:3] = draw(model, x, torch.tensor([4, 18, 48], device=cuda), uniform[0])
    assert held[:3].tolist() == first.tolist()
    u, one = uniform[1].clone(), ints([1, 1, 1, 0], cuda)

    def step():
        batch = pages.extend(seqs, one, 4, 1, 64)
        hidden = model.forward(embedding[held].to(torch.bfloat16), batch, ids)
        held.copy_(draw(model, hidden, torch.arange(4, device=cuda), u))
        return hidden
    before = [t.clone() for t in (held, *pages.state[:4])]
    step()                                                    # (warms up; then back to where it began)
    for t, b in zip((held, *pages.state[:4]), before):
        t.copy_(b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hidden = step()
    for i in range(steps):
        u.copy_(uniform[i + 1])
        graph.replay()
        assert held[:3].tolist() == want[i + 1], i
    assert torch.equal(hidden[:3], want_x)
    pages.check()
    model.check()
    assert pages.state.lens.tolist() == [lens[1] + steps, 0, lens[2] + steps, 0, lens[0] + steps, 0]
    pages.trim(seqs, ints([0, 0, 0, 0], cuda))
    assert pages.state.count.tolist() == [16, 0] and not pages.state.lens.any()


def test_a_full_cache_is_noticed_and_changes_nothing(mpq, cuda):
    weights = decoder.random_weights(CONFIG, cuda)
    model, pages = decoder.EncodedDecoder(CONFIG, weights, 4, 16), decoder.DevicePages(4, 16, 3, 4, cuda)
    x = torch.randn((50, CONFIG.width), device=cuda).to(torch.bfloat16)
    model.forward(x[:40], pages.extend(ints([0], cuda), ints([40], cuda), 40, 40, 64))
    pages.check()
    held = [t.clone() for t in model.layers[0]["cache"][:4]]
    model.forward(x, pages.extend(ints([1], cuda), ints([50], cuda), 50, 50, 64))
    with pytest.raises(MemoryError, match="3 pages are missing"):
        pages.check()
    assert all(torch.equal(a, b) for a, b in zip(held, model.layers[0]["cache"][:4]))
    pages.extend(ints([0], cuda), ints([60], cuda), 60, 60, 64)
    with pytest.raises(MemoryError, match="outgrows"):
        pages.check()
    pages.extend(ints([0], cuda), ints([3], cuda), 2, 3, 64)
    with pytest.raises(MemoryError, match="slots"):
        pages.check()
    pages.extend(ints([0], cuda), ints([3], cuda), 3, 3, 64)
    pages.check()
