"""Attention over the 4-bit cache where scores are so large that single precision holds them in steps of whole numbers and more.

Keys have one channel that is not zero, so that for half and bfloat16 queries every q . k is exact in single precision, and so is which of them is largest.  The
others are further below it than any weight reaches, or its equals, and a result is its values, or the mean of theirs: off by the rounding of the result and of
sums of up to `length` equal weights, with nothing for the exponential."""
import numpy as np
import pytest
import torch

from heads_ref import F32, KIND, attended, rounding, values_of
from test_gpu_cache_attention import run
from test_gpu_cache_attention_precision import one_channel

pytestmark = pytest.mark.gpu


def case(kind, size, scale, queries, length, seed=41):
    d, page, batch, group = 128, 16, 2, 4
    columns = -(-length // page)
    cache = one_channel(columns, page, d, seed)
    q = torch.zeros(batch, queries, group, d)
    q[..., 0] = torch.randn(batch, queries, group, generator=torch.Generator().manual_seed(seed)).sign() * torch.logspace(0, -0.3, queries * group).view(queries, group)
    q = (q * size).to(KIND[kind])
    table = torch.stack([torch.randperm(columns, generator=torch.Generator().manual_seed(i)) for i in range(batch)])
    return q, cache, table, torch.tensor([[length], [max(1, length - 7)]]), scale, page


def least_gap(q, cache, table, seen, scale, page):
    """How far below the largest score the next other one is, at least (in powers of e)"""
    k, _ = values_of(cache, page, q.shape[-1])
    least = np.inf
    for b in range(q.shape[0]):
        s = np.unique(k[table[b].numpy()][:, 0, :, 0].reshape(-1)[:int(seen[b, 0])])
        for x in q[b, :, :, 0].double().numpy().reshape(-1):
            two = np.sort(s * x * scale)[-2:]
            least = min(least, two[1] - two[0] if len(two) == 2 else np.inf)
    return least


@pytest.mark.parametrize("kind,size,scale", [("half", 60000.0, 300.0), ("half", 60000.0, -3e4), ("half", 1.0, 3e9), ("bfloat16", 1e9, 0.09), ("bfloat16", 1e12, -1.0),
                                             ("bfloat16", 1e30, 1e-10), ("bfloat16", 1e-20, 1e32), ("float", 1e10, 1.0), ("float", 1e20, 1e-5)])
@pytest.mark.parametrize("queries,length", [(1, 20), (1, 300), (1, 3000), (30, 300), (30, 3000)])
def test_the_largest_score_takes_it_all(kind, size, scale, queries, length):
    q, cache, table, seen, scale, page = case(kind, size, scale, queries, length)
    q = q if kind != "float" else q.to(torch.float16 if size < 6e4 else torch.bfloat16).float()        # (exact products)
    assert least_gap(q, cache, table, seen, scale, page) > 200
    got, lse = run(q, cache, table, seen, scale)
    k, v = values_of(cache, page, q.shape[-1])
    want, log, mean, _ = attended(q.double().numpy(), k, v, table.numpy(), np.broadcast_to(seen, q.shape[:2]), scale, 0, page)
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= rounding(kind, want) + (length + 4) * F32 * mean).all()
    assert (np.abs(lse - log) <= 6 * F32 * np.abs(log)).all()      # (the scale, the product, two sums, the factor to natural logarithms and its product)


@pytest.mark.parametrize("kind,size,scale", [("half", 60000.0, 20.0), ("half", 3000.0, 1.0), ("bfloat16", 3e6, 1.0), ("bfloat16", 2e7, 1.0), ("bfloat16", 1e8, 1.0), ("float", 3e7, 1.0)])
@pytest.mark.parametrize("queries", [1, 30])
def test_scores_of_whole_numbers(kind, size, scale, queries):
    """Steps of a quarter to eight between the scores that single precision holds: all of them in one tile or another, none of the results past the values"""
    q, cache, table, seen, scale, page = case(kind, size, scale, queries, 2000, seed=47)
    got, lse = run(q, cache, table, seen, scale)
    _, v = values_of(cache, page, q.shape[-1])
    assert np.isfinite(got).all() and np.isfinite(lse).all() and np.abs(got).max() <= np.abs(v).max() * (1 + 2.0 ** -7)
