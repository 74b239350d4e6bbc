"""The layer of examples/generate.py, prompt and tokens, against attention in 64 bits.

Bound: the keys and values that the cache holds are those of the layer itself (their rounding to four bits is another test's), the
queries those that it has rotated, so that what is left is attention: scores that are off by delta change each weight's share by exp(2 delta) at most."""
import math
import os
import sys

import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, attended, normed, rotated, rounding, values_of

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norm", [False, True])
def test_prompt_and_tokens(norm):
    from generate import Layer
    sequences, heads, kv, d, page, prompt, tokens = 3, 8, 2, 64, 16, 70, 30
    layer = Layer(sequences, prompt + tokens, heads, kv, d, page, norm=norm, stretch="linear", factor=4.0)
    qkv = torch.randn(sequences, prompt + tokens, heads + 2 * kv, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    got = [layer.prompt(qkv[:, :prompt].cuda()).cpu()]
    for i in range(prompt, prompt + tokens):
        got.append(layer.token(qkv[:, i:i + 1].cuda()).cpu().clone())
    got = torch.cat(got, 1).double().numpy()
    assert (layer.length == prompt + tokens).all()
    q = qkv[:, :, :heads].double()
    if norm:
        q = normed(q, torch.ones(d, dtype=torch.float64), 1e-6)
    freq = torch.tensor(ocn.rotary_frequencies(d, 10000.0, "linear", 4.0)[0], dtype=torch.float64)
    q = rotated(q, torch.arange(prompt + tokens).expand(sequences, -1), freq, d)[0]
    k, v = values_of(layer.cache.cpu().numpy(), page, d)
    seen = np.broadcast_to(np.arange(1, prompt + tokens + 1), (sequences, prompt + tokens))
    scale = 1 / math.sqrt(d)
    want, _, size, reach = attended(q.numpy(), k, v, layer.table.cpu().numpy(), seen, scale, 0, page)
    # a query is rounded to bfloat16 (2^-8 of each channel at most): a score is off by 2^-8 of sum |q k|
    delta = 2.0 ** -11 + 2.0 ** -21 + 2.0 ** -8 * reach + (d + 40) * F32 * (1 + reach)
    assert (np.abs(got - want) <= rounding("bfloat16", want) + np.expm1(2 * delta)[..., None] * size).all()


def test_a_layer_keeps_sequences_apart():
    """A sequence's results do not hang on what the others hold"""
    from generate import Layer
    qkv = torch.randn(2, 50, 12, 128, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).cuda()
    outs = []
    for i in range(2):
        layer = Layer(2, 60, 8, 2, 128, 16)
        x = qkv.clone()
        x[1] *= 1 + i
        outs.append((layer.prompt(x[:, :49])[0].clone(), layer.token(x[:, 49:])[0].clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_no_room():
    from generate import Layer
    layer = Layer(1, 20, 2, 1, 64, 16)
    with pytest.raises(ValueError):
        layer.prompt(torch.zeros(1, 33, 4, 64, dtype=torch.bfloat16, device="cuda"))
    layer.prompt(torch.zeros(1, 32, 4, 64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        layer.token(torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda"))
