"""Attention over the 4-bit cache against a 64-bit form on the values that the cache holds.

Bound of an output channel: half a step of its type, plus 2 delta A with A = sum p |v| / sum p and delta a weight's relative error:
the rounding of a weight (2^-11 for bfloat16 results, whose own step is 2^-8; 2^-20 for half and float), the exponential's (2^-21), the score's (D + 16 half
steps of single precision of sum |q k| scale), and the sums' (one half step for each 16 tokens)."""
import math

import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, attended, nine_bits, rounding, values_of, view

pytestmark = pytest.mark.gpu

WEIGHT = {"bfloat16": 2.0 ** -11, "half": 2.0 ** -20, "float": 2.0 ** -20}


def filled(pages, heads, page, d, seed, spread=0.5):
    """[pages, heads, block] bytes: any codes, scales around 0.15"""
    rng = np.random.default_rng(seed)
    cache = rng.integers(0, 256, (pages, heads, ocn.cache_block_bytes(page, d)), dtype=np.uint8)
    scales = nine_bits(0.15 * np.exp(spread * rng.standard_normal((pages, heads, page * d // 16))).astype(np.float32))
    cache[:, :, page * d:] = scales.view(np.uint8)
    return cache


def run(q, cache, table, seen, scale, window=0, log=True, **kw):
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device="cuda")
    lse = torch.full(q.shape[:3], 7.0, device="cuda") if log else None
    dev = [torch.as_tensor(x).cuda() for x in (cache, table, seen)]
    ocn.cache_attention(view(q.cuda()), *(view(x) for x in dev), view(out), scale, window, log_sum=None if lse is None else view(lse), **kw)
    return out.double().cpu().numpy(), None if lse is None else lse.double().cpu().numpy()


def check(kind, got, lse, q, cache, table, seen, scale, window, page):
    d = q.shape[-1]
    k, v = values_of(np.asarray(cache), page, d)
    seen = np.broadcast_to(np.asarray(seen), q.shape[:2])
    want, log, size, reach = attended(q.double().numpy(), k, v, np.asarray(table), seen, scale, window, page)
    tokens = max(1, int(seen.max())) if seen.size else 1
    score = (d + 16) * F32 * reach
    delta = WEIGHT[kind] + 2.0 ** -21 + score + (tokens / 16 + 8) * F32
    bound = rounding(kind, want) + 2 * delta[..., None] * size
    assert ((np.abs(got - want) <= bound) | (np.isnan(got) & np.isnan(want))).all(), np.nanmax(np.abs(got - want) - bound)
    if lse is not None:
        empty = np.isneginf(log)
        assert np.array_equal(np.isneginf(lse), empty)
        fine = np.isfinite(log)
        assert (np.abs(lse - log)[fine] <= (delta + 4 * F32 * np.abs(log))[fine]).all()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d,page,kv,group,queries,lengths,window", [
    (128, 16, 2, 4, 1, (1, 15, 16, 17), 0), (128, 16, 1, 8, 1, (0, 33, 257), 0), (64, 48, 3, 1, 1, (100, 47, 49), 0),
    (256, 32, 1, 5, 1, (65, 300), 0), (128, 64, 2, 16, 1, (700, 31), 0), (64, 16, 1, 20, 1, (130, 5), 0),
    (128, 32, 2, 4, 3, (2, 40, 129), 0), (64, 128, 1, 2, 17, (20, 200), 0), (128, 16, 1, 7, 40, (90, 39), 0), (256, 16, 2, 2, 9, (70,), 0),
    (128, 16, 2, 4, 1, (400, 20, 77), 33), (64, 32, 1, 3, 11, (150, 9), 16), (128, 64, 1, 8, 5, (600,), 1), (256, 64, 1, 1, 70, (75, 64), 20)])
def test_attention(d, page, kv, group, queries, lengths, window, kind):
    batch, columns = len(lengths), -(-max(lengths) // page) + 1
    pages = batch * columns + 3
    cache = filled(pages, kv, page, d, 1)
    g = torch.Generator().manual_seed(2)
    q = (torch.randn(batch, queries, kv * group, d, generator=g) * 2).to(KIND[kind])
    table = torch.randperm(pages, generator=g)[:batch * columns].view(batch, columns).to(torch.int32)
    seen = torch.tensor([[max(0, n - (queries - 1 - i)) for i in range(queries)] for n in lengths], dtype=torch.int32)
    scale = 1 / math.sqrt(d)
    got, lse = run(q, cache, table, seen, scale, window)
    check(kind, got, lse, q, cache, table, seen, scale, window, page)


@pytest.mark.parametrize("kind", ["half", "bfloat16"])
@pytest.mark.parametrize("batch,queries,length,d", [(1, 1, 5003, 128), (2, 1, 20011, 64), (1, 4, 9001, 128), (3, 150, 1500, 128), (1, 2, 3001, 256)])
def test_long(batch, queries, length, d, kind):
    """The work over one sequence in parts, and parts joined"""
    page, kv, group = 64, 2, 4
    columns = -(-length // page)
    cache = filled(batch * columns, kv, page, d, 5)
    g = torch.Generator().manual_seed(6)
    q = (torch.randn(batch, queries, kv * group, d, generator=g) * 2).to(KIND[kind])
    table = torch.randperm(batch * columns, generator=g).view(batch, columns)
    seen = torch.tensor([[length - 100 * b - (queries - 1 - i) for i in range(queries)] for b in range(batch)])
    got, lse = run(q, cache, table, seen, 0.1)
    pick = sorted({0, queries // 2, queries - 1})
    check(kind, got[:, pick], lse[:, pick], q[:, pick], cache, table, seen[:, pick], 0.1, 0, page)


def test_unseen_places_hold_anything():
    """Not-a-number scales past the end, before the window and in other pages do not reach the result; in seen places they do"""
    d, page, kv = 128, 16, 1
    cache = filled(8, kv, page, d, 1)
    table = torch.tensor([[3, 5, 0, 7]], dtype=torch.int32)
    seen = torch.tensor([[37]], dtype=torch.int32)
    clean = run(torch.ones(1, 1, 4, d).half(), cache, table, seen, 0.1, 10)
    bad = np.full_like(cache, 0xff)
    where = page * d + 2 * (np.arange(d // 16)[:, None] * page + np.arange(page))     # the places of the scales of tokens
    for token in range(27, 37):
        p, t = int(table[0, token // page]), token % page
        for c in range(d):
            wide = d // 16
            for at in (t * (d // 2) + c // 2, page * d // 2 + ((t // 4 * 16 + c // wide) * 4 + t % 4) * (wide // 2) + c % wide // 2):
                bad[p, 0, at] = cache[p, 0, at]
        for at in where[:, t]:
            bad[p, 0, at:at + 2] = cache[p, 0, at:at + 2]
    got = run(torch.ones(1, 1, 4, d).half(), bad, table, seen, 0.1, 10)
    assert np.isfinite(clean[0]).all() and np.array_equal(clean[0], got[0]) and np.array_equal(clean[1], got[1])
    p, t = int(table[0, 30 // page]), 30 % page
    bad[p, 0, where[0, t]:where[0, t] + 2] = 0xff                                    # a key's scale
    assert np.isnan(run(torch.ones(1, 1, 4, d).half(), bad, table, seen, 0.1, 10)[0]).all()


def test_pages_outside_the_cache_are_not_seen():
    d, page, kv = 64, 16, 2
    cache = filled(4, kv, page, d, 1)
    q = torch.randn(2, 2, 4, d, generator=torch.Generator().manual_seed(1)).half()
    table = torch.tensor([[1, -1, 3, 2 ** 40], [4, 99, -7, 2 ** 31]])
    seen = torch.tensor([[50, 64], [1, 64]])
    got, lse = run(q, cache, table, seen, 0.2)
    check("half", got, lse, q, cache, table, seen, 0.2, 0, page)
    assert (got[1] == 0).all() and np.isneginf(lse[1]).all()


def test_lengths_past_the_table_and_broadcast():
    d, page, kv = 128, 32, 1
    cache = filled(6, kv, page, d, 1)
    q = torch.randn(2, 3, 2, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    table = torch.tensor([[0, 1, 2], [3, 4, 5]])
    for seen in ([[5000]], [[-3]], [[70], [2 ** 40]], [[1, 2, 90]], [[-2 ** 40], [33]]):
        seen = torch.tensor(seen)
        got, lse = run(q, cache, table, seen, 0.2)
        check("bfloat16", got, lse, q, cache, table, seen, 0.2, 0, page)


@pytest.mark.parametrize("kind", list(KIND))
def test_sharp_and_flat_scores(kind):
    """One token that takes all the weight; all scores alike; large and tiny queries"""
    d, page, kv = 128, 16, 1
    cache = filled(40, kv, page, d, 4)
    table, seen = torch.arange(40)[None], torch.tensor([[640]])
    base = torch.randn(1, 1, 6, d, generator=torch.Generator().manual_seed(1))
    for size in (0.0, 1e-4, 1.0, 30.0, 3000.0):
        q = (base * size).to(KIND[kind])
        got, lse = run(q, cache, table, seen, 0.09)
        check(kind, got, lse, q, cache, table, seen, 0.09, 0, page)


def test_ranges_of_bfloat16_queries():
    d, page = 64, 16
    cache = filled(3, 1, page, d, 4)
    table, seen = torch.arange(3)[None], torch.tensor([[48]])
    base = torch.randn(1, 1, 3, d, generator=torch.Generator().manual_seed(1))
    base[0, 0, 1, ::2] *= 1e-4                   # channels of very different sizes
    for size in (1e30, 1e-30):
        q = (base * size).to(torch.bfloat16)
        got, lse = run(q, cache, table, seen, 1 / size)
        check("bfloat16", got, lse, q, cache, table, seen, 1 / size, 0, page)


def test_scales_of_any_size():
    """Keys and values from the smallest scales to the largest"""
    d, page = 64, 16
    for scale in (2.0 ** -24, 2.0 ** -15, 1.0, 5456.0):
        cache = filled(2, 1, page, d, 4)
        cache[:, :, page * d:] = np.full((2, 1, page * d // 16), scale, np.float16).view(np.uint8)
        q = torch.randn(1, 1, 4, d, generator=torch.Generator().manual_seed(1)).half()
        table, seen = torch.arange(2)[None], torch.tensor([[29]])
        got, lse = run(q, cache, table, seen, 0.1 / max(scale, 1e-3))
        check("half", got, lse, q, cache, table, seen, 0.1 / max(scale, 1e-3), 0, page)


def test_layouts_in_place_and_repeats():
    d, page, kv = 128, 16, 2
    cache = torch.from_numpy(filled(20, kv, page, d, 4)).cuda()
    wide = torch.zeros(20, kv + 1, cache.shape[2] + 128, dtype=torch.uint8, device="cuda")
    wide[:, 1:, :cache.shape[2]] = cache
    g = torch.Generator().manual_seed(1)
    q = torch.randn(2, 3, 8, d, generator=g).to(torch.bfloat16).cuda()
    table = torch.randperm(20, generator=g).view(2, 10).cuda()
    seen = torch.tensor([[150, 151, 152], [10, 11, 12]]).cuda()
    want = torch.zeros_like(q)
    ocn.cache_attention(view(q), view(cache), view(table), view(seen), view(want), 0.1)
    for layout in range(4):
        if layout == 0:
            a = q.clone()
        elif layout == 1:      # heads before queries
            a = torch.zeros(2, 8, 3, d, dtype=q.dtype, device="cuda").transpose(1, 2)
        elif layout == 2:      # channels apart
            a = torch.zeros(2, 3, 8, d, 2, dtype=q.dtype, device="cuda")[..., 0]
        else:                  # between vectors
            a = torch.zeros(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape)
        a.copy_(q)
        columns = torch.zeros(10, 2, dtype=table.dtype, device="cuda").t()
        columns.copy_(table)
        ocn.cache_attention(view(a), view(wide[:, 1:, :cache.shape[2]]), view(columns), view(seen), view(a), 0.1)
        assert torch.equal(a, want), layout


def test_side_stream_and_graph():
    d, page, kv, n = 128, 16, 2, 2000
    cache = torch.from_numpy(filled(125, kv, page, d, 4)).cuda()
    q = torch.randn(1, 1, 8, d, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    table, seen = torch.arange(125)[None].cuda(), torch.tensor([[n]]).cuda()
    want, out = torch.zeros_like(q), torch.zeros_like(q)
    v = [view(x) for x in (q, cache, table, seen, out)]
    ws = torch.empty(max(256, ocn.cache_attention_workspace_bytes(*v[:3])), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ocn.cache_attention(*v[:4], view(want), 0.1, stream=side.cuda_stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ocn.cache_attention(*v, 0.1, workspace=ws)
    for i in range(4):
        out.fill_(i)
        if i == 2:
            q.mul_(2)
            seen.fill_(1234)
            ocn.cache_attention(*v[:4], view(want), 0.1)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
