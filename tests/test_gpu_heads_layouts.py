"""Queries, keys and values in one buffer with the heads outside the tokens: normed in place, appended from it and read back into it."""
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import KIND, view

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("order", [(0, 2, 1, 3), (2, 0, 1, 3), (1, 0, 2, 3)])
def test_one_buffer_with_heads_outside(kind, order):
    batch, tokens, heads, kv, d, page = 3, 37, 6, 2, 64, 16
    g = torch.Generator().manual_seed(1)
    plain = torch.randn(batch, tokens, heads + 2 * kv, d, generator=g).to(KIND[kind]).cuda()
    buffer = plain.permute(order).contiguous()
    back = sorted(range(4), key=lambda i: order[i])
    qkv = buffer.permute(back)
    assert torch.equal(qkv, plain)
    position = torch.arange(tokens, device="cuda")
    freq = torch.tensor(ocn.rotary_frequencies(d)[0], dtype=torch.float64, device="cuda")
    rotation = ocn.Rotation(view(position), view(freq), d)
    weight = torch.rand(d, generator=g).to(KIND[kind]).cuda()

    def normed(x):
        q, k, _ = x.split([heads, kv, kv], dim=2)
        ocn.norm_rotary(view(q), view(weight), view(q), view(k), view(weight), view(k), rotation=rotation)

    normed(plain)
    normed(qkv)
    assert torch.equal(qkv, plain)
    slots = torch.randperm(batch * tokens, generator=g).view(batch, tokens).cuda()
    caches = [torch.zeros(-(-batch * tokens // page), kv, ocn.cache_block_bytes(page, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    for x, cache in zip((plain, qkv), caches):
        _, k, v = x.split([heads, kv, kv], dim=2)
        ocn.cache_append(view(k), view(v), view(slots), view(cache))
        ocn.cache_read(view(cache), view(slots), view(k), view(v))
    assert torch.equal(*caches) and torch.equal(qkv, plain)
