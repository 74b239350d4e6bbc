"""Attention over the 4-bit cache: how exactly weights are held, by type.

A result has to lie between the roundings of want - e and want + e, where want is the 64-bit form's and e = 2 delta A is what is lost before the one
rounding, with A = sum p |v| / sum p and delta as in test_gpu_cache_attention.py: a weight's error, the exponential's (2^-21), the score's ((D + 16) half steps of
single precision of sum |q k| scale) and the sums'.  A weight is off by 2^-21 of itself or less, or by 2^-36 of its row's largest where that is more, and, for half and
bfloat16, by no more than 2^-11 of itself."""
import math

import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, attended, nine_bits, values_of
from test_gpu_cache_attention import filled, run

pytestmark = pytest.mark.gpu


def outside(kind, got, q, cache, table, seen, scale, page, weight):
    """Share of the channels that are not between the two roundings"""
    d = q.shape[-1]
    k, v = values_of(cache, page, d)
    seen = np.broadcast_to(np.asarray(seen), q.shape[:2])
    want, _, size, reach = attended(q.double().numpy(), k, v, np.asarray(table), seen, scale, 0, page)
    delta = weight + 2.0 ** -21 + (d + 16) * F32 * reach + (int(seen.max()) / 16 + 8) * F32
    # (rounding twice, to single precision and then to the type, is not rounding once within 2^-24 of a tie)
    e = 2 * delta[..., None] * size + F32 * np.abs(want)
    ends = [torch.from_numpy(want + s * e).to(KIND[kind]).double().numpy() for s in (-1, 1)]
    return 1 - ((ends[0] <= got) & (got <= ends[1])).mean()


def one_channel(pages, page, d, seed):
    """A cache whose keys have one channel that is not zero, of any size up to 12 / 8, so that scores are exact but for their last rounding"""
    cache = filled(pages, 1, page, d, seed)
    rng = np.random.default_rng(seed + 1)
    cache[:, :, :page * d // 2] = 0
    cache[:, :, :page * d // 2:d // 2] = rng.integers(0, 16, (pages, 1, page))
    scales = nine_bits(rng.uniform(1 / 16, 1 / 8, (pages, 1, page * d // 32)).astype(np.float32))
    cache[:, :, page * d:page * d + page * d // 16] = scales.view(np.uint8)
    return cache


def one_rounding_case(kind, d, queries, length):
    page, pages, group = 16, 12, 4
    cache = one_channel(pages, page, d, 31 + length)
    q = torch.zeros(6, queries, group, d)
    q[..., 0] = torch.randn(6, queries, group, generator=torch.Generator().manual_seed(32))
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(33)).view(6, 2)
    return q.to(KIND[kind]), cache, table, torch.full((6, 1), length), 1.0, page


@pytest.mark.parametrize("kind", ["half", "bfloat16"])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("length", [2, 3, 5, 8, 13, 32])
def test_one_rounding(kind, d, queries, length):
    """Few tokens of weights alike: a weight's own rounding to the type's size would reach the result"""
    q, cache, table, seen, scale, page = one_rounding_case(kind, d, queries, length)
    got, _ = run(q, cache, table, seen, scale)
    assert outside(kind, got, q, cache, table, seen, scale, page, 2.0 ** -21) == 0


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("queries", [1, 20])
@pytest.mark.parametrize("bits", [8.0, 13.5, 14.5, 16.0, 19.0, 22.0, 24.5, 25.5, 40.0, 52.0, 54.0, 80.0, 110.0])
def test_channels_of_light_tokens_alone(kind, queries, bits):
    """Values that are zero in the tokens with large weights: what others give them, `bits` powers of two below"""
    d, page, group, length = 128, 16, 4, 96
    cache = filled(length // page, 1, page, d, 23)
    # keys: +-1 in one channel, which every query has; values: nothing in the even channels of every heavy token
    cache[:, :, :page * d // 2] = 0
    cache[:, :, page * d:page * d + page * d // 16] = nine_bits(np.ones((length // page, 1, page * d // 32), np.float32)).view(np.uint8)
    heavy = np.arange(length) % 3 == 0
    for token in range(length):
        block = cache[token // page, 0]
        block[token % page * (d // 2)] = 0x1 if heavy[token] else 0x9
        if heavy[token]:
            at, wide = token % page, d // 16
            for c in range(0, d, 2):
                block[page * d // 2 + ((at // 4 * 16 + c // wide) * 4 + at % 4) * (wide // 2) + c % wide // 2] &= 0xf0
    q = torch.zeros(1, queries, group, d)
    q[..., 0] = 1
    q = q.to(KIND[kind])
    table, seen = torch.arange(length // page)[None], torch.tensor([[length]])
    scale = bits * math.log(2) / 2                 # scores of +-1 times this
    got, _ = run(q, cache, table, seen, scale)
    weight = max(2.0 ** -21, min(2.0 ** -36 * 2.0 ** bits, 2.0 ** -21 if kind == "float" else 2.0 ** -11))
    assert kind == "half" or (got[..., ::2] != 0).any()      # (of half they are its smallest numbers, or zero)
    assert outside(kind, got, q, cache, table, seen, scale, page, weight) == 0
