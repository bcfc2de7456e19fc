"""The decoder of encoded layers: the block's operators run together, against the same network in 64 bits, and with
itself when the same tokens come as whole prompts, in chunks and one by one; the host's side of the cache on the CPU."""
import math

import pytest
import torch

from paper_1905_13389_b200 import decoder

CONFIG = decoder.Config(layers=2, width=256, heads=8, kv_heads=2, dim=64, inner=768)


def reference(config, weights, x, lens):
    """The network in 64 bits without any quantization, sequences one after the other in x."""
    x = x.double()
    for w in weights:
        w = {k: v.double() for k, v in w.items()}
        norm = lambda t, g: t / torch.sqrt((t * t).mean(1, keepdim=True) + config.eps) * g      # noqa: E731
        q, k, v = (norm(x, w["norm1"]) @ w["qkv"].T).view(x.shape[0], -1, config.dim).split((config.heads, config.kv_heads, config.kv_heads), 1)
        k, v = (t.repeat_interleave(config.heads // config.kv_heads, 1) for t in (k, v))
        parts, at = [], 0
        for n in lens:
            s = torch.einsum("ihd,jhd->hij", q[at:at + n], k[at:at + n]) / math.sqrt(config.dim)
            s = s.masked_fill(torch.ones((n, n), dtype=torch.bool, device=x.device).triu(1), -math.inf)
            parts.append(torch.einsum("hij,jhd->ihd", torch.softmax(s, -1), v[at:at + n]).flatten(1))
            at += n
        x = x + torch.cat(parts) @ w["o"].T
        h = torch.nn.functional.gelu(norm(x, w["norm2"]) @ w["up"].T + w["up_bias"], approximate="tanh")
        x = x + h @ w["down"].T
    return x


def relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.gpu
@pytest.mark.parametrize("cache_bits", [8, 4])
def test_against_64_bits(mpq, cuda, cache_bits):
    """An operand of 8 bits with the range of its row is off by a uniform error of a step 2s/255: with s about 3.5 times
    the row's root mean square 0.8 % of it.  A product has two such operands, a block four products and the cache between
    (7.5 times that error per key and value with 4 bits, of which the softmax averages most): 5 % and 15 % of the result
    leave a factor of two over two blocks' errors added as if they never cancelled."""
    config = CONFIG._replace(cache_bits=cache_bits)
    weights = decoder.random_weights(config, cuda)
    model = decoder.EncodedDecoder(config, weights, pages=32, page_size=16)
    lens = {0: 70, 1: 1, 2: 33}
    x = torch.randn((sum(lens.values()), config.width), generator=torch.Generator().manual_seed(2)).to(cuda).to(torch.bfloat16)
    got = model.forward(x, decoder.Pages(32, 16).extend(lens, cuda))
    assert relative(got, reference(config, weights, x, lens.values())) < (0.05 if cache_bits == 8 else 0.15)


@pytest.mark.gpu
def test_chunks_and_single_tokens_give_what_whole_prompts_give(mpq, cuda):
    """The same arithmetic per token however it is batched, except for the order of sums inside the attention: a few
    roundings of bfloat16 (2^-9 each), some of which move a level of the next operand by one step."""
    weights = decoder.random_weights(CONFIG, cuda)
    x = {s: torch.randn((n, CONFIG.width), generator=torch.Generator().manual_seed(s)).to(cuda).to(torch.bfloat16) for s, n in ((0, 60), (1, 45))}

    def run(steps):
        model, pages = decoder.EncodedDecoder(CONFIG, weights, pages=16, page_size=8), decoder.Pages(16, 8)
        out, at = {0: [], 1: []}, {0: 0, 1: 0}
        for step in steps:
            y = model.forward(torch.cat([x[s][at[s]:at[s] + n] for s, n in step.items()]), pages.extend(step, cuda))
            for s, part in zip(step, y.split(list(step.values()))):
                out[s].append(part)
                at[s] += step[s]
        return torch.cat(out[0] + out[1])
    whole = run([{0: 60, 1: 45}])
    assert relative(run([{1: 20}, {0: 33, 1: 24}, {1: 1, 0: 27}]), whole) < 0.02
    assert relative(run([{0: 50, 1: 40}] + [{0: 1, 1: 1}] * 5 + [{0: 1}] * 5), whole) < 0.02


@pytest.mark.gpu
def test_a_step_can_be_captured_in_a_graph(mpq, cuda):
    weights = decoder.random_weights(CONFIG, cuda)
    model, pages = decoder.EncodedDecoder(CONFIG, weights, pages=16, page_size=16), decoder.Pages(16, 16)
    x = torch.randn((40, CONFIG.width), device=cuda).to(torch.bfloat16)
    model.forward(x, pages.extend({0: 40}, cuda))
    batch, token = pages.extend({0: 1}, cuda), torch.randn((1, CONFIG.width), device=cuda).to(torch.bfloat16)
    ref = model.forward(token, batch).clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = model.forward(token, batch)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, ref)


@pytest.mark.gpu
def test_the_demo_runs(mpq, cuda, capsys):
    decoder.main()
    assert "sequence 1, 12 tokens in the cache" in capsys.readouterr().out


def test_pages():
    pages = decoder.Pages(6, 4)
    b = pages.extend({7: 5, 3: 4}, "cpu")
    assert b.q_starts.tolist() == [0, 5, 9] and b.kv_lens.tolist() == [5, 4] and b.max_q == 5 and b.max_kv == 5
    assert b.table.tolist() == [[0, 1], [2, 0]] and b.slots.tolist() == [0, 1, 2, 3, 4, 8, 9, 10, 11]
    b = pages.extend({3: 1, 7: 3}, "cpu")
    assert b.table.tolist() == [[2, 3], [0, 1]] and b.slots.tolist() == [12, 5, 6, 7] and b.kv_lens.tolist() == [5, 8]
    with pytest.raises(MemoryError):
        pages.extend({9: 12}, "cpu")
    assert 9 not in pages.owned and len(pages.free) == 2        # nothing was taken
    pages.drop(7)
    assert pages.extend({9: 12}, "cpu").slots.tolist() == [j for p in (1, 0, 4) for j in range(4 * p, 4 * p + 4)]
