"""Attention over the 4-bit cache where many rows share a head of the cache, in caches past 4 GB, in several launches, of nothing, and
with appending in one graph.  Bounds as in test_gpu_cache_attention.py."""
import math

import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import KIND, held, view
from test_gpu_cache_attention import check, filled, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d,page,kv,group,queries,lengths,window", [
    (64, 16, 2, 8, 30, (90, 31, 0), 0), (64, 48, 1, 1, 130, (200, 64), 17), (64, 128, 3, 5, 33, (129,), 0), (128, 32, 1, 4, 70, (100, 69, 1), 40),
    (128, 16, 2, 65, 1, (33, 7), 0), (128, 48, 1, 3, 43, (500,), 1), (256, 64, 1, 9, 15, (300, 2), 0), (256, 16, 2, 13, 5, (31, 32, 33), 9)])
def test_many_rows(d, page, kv, group, queries, lengths, window, kind):
    """More than 64 rows to a head of the cache: every size of head and type, blocks of rows that end inside, rows that see nothing"""
    batch, columns = len(lengths), -(-max(lengths) // page) + 1
    pages = batch * columns + 3
    cache = filled(pages, kv, page, d, 11)
    g = torch.Generator().manual_seed(12)
    q = (torch.randn(batch, queries, kv * group, d, generator=g) * 2).to(KIND[kind])
    table = torch.randperm(pages, generator=g)[:batch * columns].view(batch, columns).to(torch.int32)
    table[0, 0] = -1 if len(lengths) == 3 else table[0, 0]
    seen = torch.tensor([[max(0, n - (queries - 1 - i)) for i in range(queries)] for n in lengths], dtype=torch.int32)
    scale = 1 / math.sqrt(d)
    got, lse = run(q, cache, table, seen, scale, window)
    check(kind, got, lse, q, cache, table, seen, scale, window, page)


def put_nan(cache, page, d, token, v):
    """Not a number as the scales of a token's keys or values in a block"""
    at = page * d + (d // 16 * page if v else 0) + 2 * (np.arange(d // 32) * page + token)
    cache[at] = 0xff
    cache[at + 1] = 0x7f


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("queries", [6, 90])
def test_scales_that_are_not_numbers_reach_the_rows_that_see_them(d, queries):
    page, n = 16, 150
    columns = -(-n // page)
    cache = filled(columns, 1, page, d, 3)
    g = torch.Generator().manual_seed(4)
    q = torch.randn(1, queries, 2, d, generator=g).to(torch.bfloat16)
    table = torch.randperm(columns, generator=g)[None]
    seen = torch.tensor([[n - (queries - 1 - i) for i in range(queries)]])
    clean, clean_log = run(q, cache, table, seen, 0.1, 40)
    token = n - 2      # seen by the last two queries
    for v in (False, True):
        bad = cache.copy()
        put_nan(bad[int(table[0, token // page]), 0], page, d, token % page, v)
        got, log = run(q, bad, table, seen, 0.1, 40)
        assert np.array_equal(got[:, :-2], clean[:, :-2]) and np.isnan(got[:, -2:]).all()
        assert np.array_equal(log[:, :-2], clean_log[:, :-2])


def test_a_cache_past_4_gb():
    """Pages at the end of 5.5 GB: appended to, read back and attended to"""
    d, page, kv = 128, 64, 2
    pages = 300001
    cache = torch.empty(pages, kv, ocn.cache_block_bytes(page, d), dtype=torch.uint8, device="cuda")
    where = torch.tensor([[pages - 1, 0, pages - 2, 250000]])
    n = 230
    slots = (where[0, torch.arange(n) // page] * page + torch.arange(n) % page).to(torch.int32)
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn(n, kv, d, generator=g).half() for _ in range(2))
    ocn.cache_append(view(k.cuda()), view(v.cuda()), view(slots.cuda()), view(cache))
    back = [torch.zeros_like(k).cuda() for _ in range(2)]
    ocn.cache_read(view(cache), view(slots.cuda()), view(back[0]), view(back[1]))
    for x, y in zip((k, v), back):
        assert np.array_equal(y.double().cpu().numpy(), held(x.double().numpy()))
    small = cache[where[0].cuda()].cpu().numpy()
    for queries in (1, 40):
        q = torch.randn(1, queries, 8, d, generator=g).half()
        seen = torch.full((1, queries), n)
        got, lse = run(q, cache, where, seen, 0.1)
        check("half", got, lse, q, small, torch.arange(4)[None], seen, 0.1, 0, page)


def test_slots_past_32_bits():
    """One block's bytes as every page of 2^28: slots of more than 31 bits"""
    d, page = 64, 16
    block = torch.from_numpy(filled(1, 1, page, d, 7)).cuda()
    pages = 1 << 28
    cache = ocn.Tensor(block.data_ptr(), "uint8", (pages, 1, block.shape[2]), (0, 0, 1), 0, 0, block)
    slots = torch.tensor([3, 2 ** 31 + 5, pages * page - 1, pages * page, 2 ** 62])
    k, v = (torch.full((5, 1, d), 9.0, device="cuda") for _ in range(2))
    ocn.cache_read(cache, view(slots.cuda()), view(k), view(v))
    want = [torch.full((5, 1, d), 9.0, device="cuda") for _ in range(2)]
    ocn.cache_read(view(block), view(torch.tensor([3, 5, 15, -1, -1]).cuda()), view(want[0]), view(want[1]))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


@pytest.mark.parametrize("queries,columns", [(1, 4), (1, 60), (3, 60), (40, 4), (40, 60)])
def test_several_launches(queries, columns):
    """Workgroups of one call in launches of three"""
    from paper_1810_08723_amd import binding
    d, page, kv, batch = 128, 32, 2, 3
    cache = filled(columns * batch, kv, page, d, 2)
    g = torch.Generator().manual_seed(3)
    q = torch.randn(batch, queries, 8, d, generator=g).half()
    table = torch.randperm(columns * batch, generator=g).view(batch, columns)
    seen = torch.tensor([[columns * page - 5], [17], [columns * page]])
    want = run(q, cache, table, seen, 0.1)
    k, v = (torch.randn(batch * 37, kv, d, generator=g).half().cuda() for _ in range(2))
    slots = torch.randperm(columns * batch * page, generator=g)[:batch * 37].cuda()
    caches = [torch.zeros(columns * batch, kv, cache.shape[2], dtype=torch.uint8, device="cuda") for _ in range(2)]
    back = [torch.zeros_like(k) for _ in range(4)]
    ocn.cache_append(view(k), view(v), view(slots), view(caches[0]))
    ocn.cache_read(view(caches[0]), view(slots), view(back[0]), view(back[1]))
    binding.set_max_launch_blocks(3)
    try:
        got = run(q, cache, table, seen, 0.1)
        ocn.cache_append(view(k), view(v), view(slots), view(caches[1]))
        ocn.cache_read(view(caches[1]), view(slots), view(back[2]), view(back[3]))
        torch.cuda.synchronize()
    finally:
        binding.set_max_launch_blocks(0)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    assert torch.equal(caches[0], caches[1]) and torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])


def test_nothing_to_do_and_nothing_to_see():
    d, page = 64, 16
    cache = filled(3, 2, page, d, 1)
    for shape in ((0, 1, 4, d), (2, 0, 4, d), (2, 3, 0, d)):
        q = torch.zeros(shape).half()
        out, _ = run(q, cache, torch.zeros(shape[0], 2, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32), 0.1)
        assert out.shape == shape
    for queries in (2, 50):
        q = torch.randn(2, queries, 4, d).half()
        for held_cache, columns in ((cache, 0), (cache[:0], 2)):     # a table without columns, a cache without pages
            out, lse = run(q, held_cache, torch.zeros(2, columns, dtype=torch.int64), torch.full((2, 1), 20), 0.1)
            assert (out == 0).all() and np.isneginf(lse).all()
    empty = torch.zeros(0, 2, d).half().cuda()
    ocn.cache_append(view(empty), view(empty), view(torch.zeros(0, dtype=torch.int64).cuda()), view(torch.from_numpy(cache).cuda()))


def test_a_step_of_generation_in_a_graph():
    """Norm with rotation, appending and attention, captured once and replayed for tokens that follow each other"""
    d, page, kv, heads, batch, first = 128, 16, 2, 8, 3, 300
    g = torch.Generator().manual_seed(1)
    columns = first // page + 4
    cache = torch.from_numpy(filled(batch * columns, kv, page, d, 6)).cuda()
    other = cache.clone()
    table = torch.randperm(batch * columns, generator=g).view(batch, columns).to(torch.int32).cuda()
    freq = torch.tensor(ocn.rotary_frequencies(d)[0], dtype=torch.float64, device="cuda")
    qkv = torch.zeros(batch, 1, heads + 2 * kv, d, dtype=torch.bfloat16, device="cuda")
    position, slots, seen = (torch.zeros(batch, 1, dtype=torch.int32, device="cuda") for _ in range(3))
    weight = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    out = torch.zeros(batch, 1, heads, d, dtype=torch.bfloat16, device="cuda")
    want = torch.zeros_like(out)
    q, k, v = qkv[:, :, :heads], qkv[:, :, heads:heads + kv], qkv[:, :, heads + kv:]
    rotation = ocn.Rotation(view(position), view(freq), d)
    ws = torch.empty(max(256, ocn.cache_attention_workspace_bytes(view(q), view(cache), view(table))), dtype=torch.uint8, device="cuda")

    def step(to, result):
        ocn.norm_rotary(view(q), view(weight), view(q), view(k), view(weight), view(k), rotation=rotation)
        ocn.cache_append(view(k), view(v), view(slots), view(to))
        ocn.cache_attention(view(q), view(to), view(table), view(seen), view(result), 0.1, workspace=ws)

    slots.fill_(-1)
    step(other, want)            # (nothing is appended: kernels are loaded before they are captured)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(cache, out)
    for i in range(20):
        new = torch.randn(qkv.shape, generator=g).to(torch.bfloat16).cuda()
        at = first + i
        position.fill_(at)
        seen.fill_(at + 1)
        slots.copy_(table[:, at // page, None] * page + at % page)
        qkv.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        qkv.copy_(new)
        step(other, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache, other), i


def test_gradient_of_the_norm_in_a_graph():
    d, heads, kv, tokens = 128, 6, 2, 700
    g = torch.Generator().manual_seed(1)
    make = lambda n: torch.randn(tokens, n, d, generator=g).half().cuda()  # noqa: E731
    q, k, qg, kg = make(heads), make(kv), make(heads), make(kv)
    weight = torch.rand(d, generator=g).cuda()
    freq = torch.tensor(ocn.rotary_frequencies(d)[0], dtype=torch.float64, device="cuda")
    position = torch.arange(tokens, device="cuda")
    rotation = ocn.Rotation(view(position), view(freq), d)
    outs = [[torch.zeros_like(q), torch.zeros(d, device="cuda"), torch.zeros_like(k), torch.zeros(d, device="cuda")] for _ in range(2)]
    ws = torch.empty(ocn.norm_rotary_grad_workspace_bytes(view(q), view(k)), dtype=torch.uint8, device="cuda")

    def step(o):
        ocn.norm_rotary_grad(view(qg), view(q), view(weight), view(o[0]), view(o[1]), view(kg), view(k), view(weight), view(o[2]), view(o[3]),
                             rotation=rotation, workspace=ws)

    step(outs[1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(outs[0])
    for i in range(4):
        qg.mul_(1.0 + i)
        position.add_(i)
        for o in outs[0]:
            o.fill_(float(i))
        graph.replay()
        step(outs[1])
        torch.cuda.synchronize()
        for a, b in zip(*outs):
            assert torch.equal(a, b), i


def test_several_launches_of_many_rows():
    """As above, with so many rows that a wavefront joins each"""
    test_several_launches(60, 60)
