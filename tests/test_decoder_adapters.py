"""Adapters that do not fit the decoder they are given to, on a machine without a GPU."""
import pytest
import torch

from paper_1905_13389_b200 import decoder

CONFIG = decoder.Config(layers=3, width=32, heads=2, kv_heads=1, dim=64, inner=48)


def test_adapters_are_given_for_every_layer_and_for_its_products():
    weights, low = decoder.random_weights(CONFIG, "cpu"), decoder.random_adapters(CONFIG, 2, 4, "cpu")
    for bad in (low[:2], low + low[:1]):
        with pytest.raises(ValueError, match="3 layers"):
            decoder.EncodedDecoder(CONFIG, weights, 4, 16, bad)
    with pytest.raises(ValueError, match="'gate'"):
        decoder.EncodedDecoder(CONFIG, weights, 4, 16, [dict(low[0], gate=low[0]["up"]), {}, {}])


def test_adapters_of_other_sizes_than_the_product():
    weights, low = decoder.random_weights(CONFIG, "cpu"), decoder.random_adapters(CONFIG, 2, 4, "cpu")
    for name, other in (("up", "down"), ("qkv", "up"), ("down", "o")):
        with pytest.raises(ValueError, match=name):
            decoder.EncodedDecoder(CONFIG, weights, 4, 16, [{}, {name: low[1][other]}, {}])
