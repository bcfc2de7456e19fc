"""Decoder of encoded layers that serves tokens (driver; every step of a block runs in libmpq's kernels).

A block is the usual one of a decoder-only transformer, with every product on levels:

    h   = x (+ the block before's output)                       rmsnorm_levels   (adds, normalizes, encodes)
    qkv = h W_qkv                                               linear_levels
    keys and values -> paged cache on 8- or 4-bit levels        cache_write
    a   = attention of the new tokens over the cache            cache_attention
    x   = x + encode(a) W_o                                     encode_levels, linear_levels (residual in its store)
    h   = x                                                     rmsnorm_levels
    x   = x + encode(gelu(h W_up + b_up)) W_down                linear_levels (bias, GELU), encode_levels, linear_levels

Weights are encoded once, at construction, with one range per output channel; activations get one range per
token.  Positions are the caller's to put into the hidden states.  ``forward`` takes the new tokens of a batch of
sequences -- whole prompts, chunks of prompts and single tokens mixed -- and only launches kernels on the current
stream; ``check`` says afterwards whether all of them have done their work.  ``Pages`` keeps the host's side of the cache: which pages a sequence owns.

    python -m paper_1905_13389_b200.decoder          # a small model: two prompts, then eight tokens each
"""
from __future__ import annotations

from typing import Dict, List, NamedTuple

import torch

from . import binding as mpq


class Config(NamedTuple):
    layers: int
    width: int                    # of the hidden states
    heads: int
    kv_heads: int
    dim: int                      # of a head
    inner: int                    # of the feed-forward part
    weight_bits: int = 8
    act_bits: int = 8
    cache_bits: int = 8
    eps: float = 1e-6


class Batch(NamedTuple):
    """New tokens of some sequences, as the cache calls take them (device tensors, and the launch bounds)."""
    slots: torch.Tensor
    q_starts: torch.Tensor
    kv_lens: torch.Tensor
    table: torch.Tensor
    max_q: int
    max_kv: int


class Pages:
    """Which pages of a cache each sequence owns; pages are taken as sequences grow and given back by ``drop``."""

    def __init__(self, pages: int, page_size: int):
        self.page_size, self.free = page_size, list(range(pages))[::-1]
        self.owned: Dict[int, List[int]] = {}
        self.length: Dict[int, int] = {}

    def extend(self, tokens: Dict[int, int], device) -> Batch:
        """Makes room for tokens[s] new tokens of each sequence s (in the dict's order) and describes the batch."""
        need = {s: -(-(self.length.get(s, 0) + n) // self.page_size) - len(self.owned.get(s, [])) for s, n in tokens.items()}
        if sum(need.values()) > len(self.free):
            raise MemoryError("the cache is full: %d pages wanted, %d free" % (sum(need.values()), len(self.free)))
        slots, starts, lens = [], [0], []
        for s, n in tokens.items():
            mine = self.owned.setdefault(s, [])
            mine += [self.free.pop() for _ in range(need[s])]
            old = self.length.get(s, 0)
            slots += [mine[j // self.page_size] * self.page_size + j % self.page_size for j in range(old, old + n)]
            self.length[s] = old + n
            starts.append(starts[-1] + n)
            lens.append(old + n)
        per = max(1, max(len(self.owned[s]) for s in tokens))
        table = [self.owned[s] + [0] * (per - len(self.owned[s])) for s in tokens]
        to = lambda v, dtype: torch.tensor(v, dtype=dtype).to(device)                          # noqa: E731
        return Batch(to(slots, torch.int64), to(starts, torch.int32), to(lens, torch.int32), to(table, torch.int32),
                     max(tokens.values()), max(lens))

    def drop(self, sequence: int):
        self.free += self.owned.pop(sequence, [])
        self.length.pop(sequence, None)


class EncodedDecoder:
    """``weights``: per layer a dict of float tensors qkv [(heads + 2 kv_heads) dim x width], o [width x heads dim],
    up [inner x width], up_bias [inner], down [width x inner], norm1, norm2 [width]."""

    def __init__(self, config: Config, weights: List[Dict[str, torch.Tensor]], pages: int, page_size: int):
        self.config, device = config, weights[0]["qkv"].device
        self.layers = []
        for w in weights:
            layer = {name: mpq.encode_levels(w[name], config.weight_bits) for name in ("qkv", "o", "up", "down")}
            layer.update({name: w[name].float().contiguous() for name in ("up_bias", "norm1", "norm2")})
            layer["cache"] = mpq.level_cache(pages, config.kv_heads, page_size, config.dim, config.cache_bits, device)
            self.layers.append(layer)
        self.given_up = mpq.wait_failures()

    def forward(self, x: torch.Tensor, batch: Batch) -> torch.Tensor:
        """Hidden states [tokens][width] (float16 or bfloat16) of the batch's new tokens -> hidden states after the last
        block; the tokens' keys and values are in the cache afterwards."""
        c, dtype = self.config, x.dtype
        tokens = x.shape[0]
        for w in self.layers:
            h = mpq.rmsnorm_levels(x, w["norm1"], c.eps, c.act_bits)
            qkv = mpq.linear_levels(h, w["qkv"], dtype=dtype).view(tokens, c.heads + 2 * c.kv_heads, c.dim)
            q, k, v = qkv.split((c.heads, c.kv_heads, c.kv_heads), dim=1)
            mpq.cache_write(w["cache"], k, v, batch.slots)
            a = mpq.cache_attention(q, w["cache"], batch.q_starts, batch.kv_lens, batch.table, batch.max_q, batch.max_kv)
            a = mpq.encode_levels(a.view(tokens, c.heads * c.dim), c.act_bits)
            x = mpq.linear_levels(a, w["o"], residual=x, dtype=dtype)
            h = mpq.rmsnorm_levels(x, w["norm2"], c.eps, c.act_bits)
            h = mpq.linear_levels(h, w["up"], bias=w["up_bias"], act="gelu_tanh", dtype=dtype)
            x = mpq.linear_levels(mpq.encode_levels(h, c.act_bits), w["down"], residual=x, dtype=dtype)
        return x


    def check(self):
        """Raises if a kernel has given up a wait since the model was made or last checked.  What it left is NaN, but an encoder
        behind it takes a NaN for a zero, so the hidden states need not show it.  Waits for the stream: for a place where the
        caller waits for a result anyway."""
        before, self.given_up = self.given_up, mpq.wait_failures()
        if self.given_up != before:
            raise RuntimeError("%d CTAs gave up a wait: the results since the last check are not valid" % (self.given_up - before))


def random_weights(config: Config, device, seed: int = 0) -> List[Dict[str, torch.Tensor]]:
    g = torch.Generator().manual_seed(seed)
    normal = lambda n, k: (torch.randn((n, k), generator=g) / k ** 0.5).to(device)             # noqa: E731
    out = []
    for _ in range(config.layers):
        out.append({"qkv": normal((config.heads + 2 * config.kv_heads) * config.dim, config.width), "o": normal(config.width, config.heads * config.dim),
                    "up": normal(config.inner, config.width), "down": normal(config.width, config.inner),
                    "up_bias": (0.1 * torch.randn((config.inner,), generator=g)).to(device),
                    "norm1": (1 + 0.1 * torch.randn((config.width,), generator=g)).to(device),
                    "norm2": (1 + 0.1 * torch.randn((config.width,), generator=g)).to(device)})
    return out


def main():
    device = torch.device("cuda:0")
    config = Config(layers=4, width=1024, heads=16, kv_heads=4, dim=64, inner=4096)
    model = EncodedDecoder(config, random_weights(config, device), pages=64, page_size=16)
    pages, g = Pages(64, 16), torch.Generator().manual_seed(1)
    vocabulary = torch.randn((500, config.width), generator=g).to(device)
    words = mpq.encode_levels(vocabulary, 8)                 # the last product is on levels as well
    tokens = {0: torch.randint(0, 500, (37,), generator=g), 1: torch.randint(0, 500, (5,), generator=g)}
    said = {s: [] for s in tokens}
    for _ in range(8):
        batch = pages.extend({s: len(t) for s, t in tokens.items()}, device)
        x = vocabulary[torch.cat(list(tokens.values())).to(device)].to(torch.bfloat16)
        x = model.forward(x, batch)[batch.q_starts[1:].long() - 1]                             # each sequence's last token
        logits = mpq.linear_levels(mpq.rmsnorm_levels(x, None, config.eps), words)
        nxt = logits.argmax(1).cpu()
        model.check()
        tokens = {s: nxt[i:i + 1] for i, s in enumerate(tokens)}
        for i, s in enumerate(said):
            said[s].append(int(nxt[i]))
    for s, t in said.items():
        print("sequence %d, %d tokens in the cache: %s" % (s, pages.length[s], t))
        pages.drop(s)


if __name__ == "__main__":
    main()
