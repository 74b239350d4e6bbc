"""Attention over the 4-bit cache: queries and results of any layout, and in one place, in every kernel that reads and writes them (few and many rows, in one part and in
several, parts joined by a workgroup and by a wavefront); peaked scores with many rows.  Bits against a call with contiguous tensors, and that against the 64-bit form."""
import math

import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, attended, rounding, values_of, view
from test_gpu_cache_attention import WEIGHT, check, filled, run

pytestmark = pytest.mark.gpu


def laid(x, layout):
    """x [batch, queries, heads, channels] in other places"""
    b, t, h, d = x.shape
    new = lambda *s: torch.zeros(*s, dtype=x.dtype, device=x.device)  # noqa: E731
    y = {"heads first": lambda: new(b, h, t, d).transpose(1, 2), "in a wider row": lambda: new(b, t, h + 3, d + 16)[:, :, 2:h + 2, 8:d + 8],
         "channels apart": lambda: new(b, t, h, d, 3)[..., 1], "channels outermost": lambda: new(d, b, t, h).permute(1, 2, 3, 0),
         "between vectors": lambda: new(b * t * h * d + 1)[1:].view(b, t, h, d), "last sequence first": lambda: new(b, t, h, d)}[layout]()
    return y.copy_(x)


def reversed_view(y):
    """The descriptor that goes through y's sequences backwards"""
    v = view(y)
    return ocn.Tensor(v.base, v.dtype, v.sizes, (-v.strides[0],) + v.strides[1:], v.offset + (y.shape[0] - 1) * v.strides[0], v.device, y)


SHAPES = {"few rows": (2, 3, 4, 160), "few rows in parts": (2, 1, 4, 3000), "few rows in parts, joined by wavefronts": (64, 2, 4, 1500), "many rows": (2, 30, 4, 160),
          "many rows in parts": (2, 30, 4, 3000), "many rows in parts, joined by wavefronts": (3, 100, 4, 2000), "32 rows in parts": (2, 8, 4, 2000)}


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("shape", list(SHAPES))
def test_layouts_and_in_place(shape, d, kind):
    batch, queries, group, length = SHAPES[shape]
    page, kv, pages = 32, 2, 40
    g = torch.Generator().manual_seed(1)
    cache = torch.from_numpy(filled(pages, kv, page, d, 4)).cuda()
    q = torch.randn(batch, queries, kv * group, d, generator=g).to(KIND[kind]).cuda()
    table = torch.randint(0, pages, (batch, -(-length // page)), generator=g).cuda()
    seen = (torch.arange(length - queries + 1, length + 1)[None] - 5 * torch.arange(batch)[:, None]).clamp(min=0).cuda()
    want, log = torch.zeros_like(q), torch.zeros(q.shape[:3], device="cuda")
    ocn.cache_attention(view(q), view(cache), view(table), view(seen), view(want), 0.1, log_sum=view(log))
    need = ocn.cache_attention_workspace_bytes(view(q), view(cache), view(table))
    assert (need > 0) == ("parts" in shape)
    for layout in ("heads first", "in a wider row", "channels apart", "channels outermost", "between vectors", "last sequence first"):
        a, out = laid(q, layout), laid(torch.zeros_like(q), layout)
        flip = layout == "last sequence first"
        logs = torch.zeros(*q.shape[:3], 2, device="cuda")[..., 1]
        ocn.cache_attention(view(a), view(cache), view(table), view(seen), view(out), 0.1, log_sum=view(logs))
        assert torch.equal(out, want) and torch.equal(logs, log), layout
        if flip:
            a, out = a.flip(0).contiguous(), torch.zeros_like(out)
            ocn.cache_attention(reversed_view(a), view(cache), view(table), view(seen), reversed_view(out), 0.1)
            assert torch.equal(out.flip(0), want), layout
        v = reversed_view(a) if flip else view(a)
        ocn.cache_attention(v, view(cache), view(table), view(seen), v, 0.1)
        assert torch.equal(a.flip(0) if flip else a, want), ("in place", layout)
    pick = sorted({0, queries - 1})
    check(kind, want[:2, pick].double().cpu().numpy(), log[:2, pick].double().cpu().numpy(), q[:2, pick].cpu(), cache.cpu().numpy(), table[:2].cpu(), seen[:2, pick].cpu(),
          0.1, 0, page)


def check_far(kind, got, lse, q, cache, table, seen, scale, page):
    """As check(), where weights may be too small for single precision: those below 2^-122 of a row's largest are zero or not, each worth that much of its value"""
    d = q.shape[-1]
    k, v = values_of(cache, page, d)
    seen = np.broadcast_to(np.asarray(seen), q.shape[:2])
    want, log, size, reach = attended(q.double().numpy(), k, v, np.asarray(table), seen, scale, 0, page)
    delta = WEIGHT[kind] + 2.0 ** -21 + (d + 16) * F32 * reach + (int(seen.max()) / 16 + 8) * F32
    bound = rounding(kind, want) + 2 * delta[..., None] * size + 2.0 ** -122 * int(seen.max()) * np.abs(v).max()
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) - bound).max()
    assert (np.abs(lse - log) <= delta + 4 * F32 * np.abs(log)).all()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("size", [0.0, 1e-4, 3.0, 30.0, 3000.0])
def test_peaked_and_flat_scores_of_many_rows(kind, d, size):
    """One token that takes all the weight; all scores alike; weights below the smallest that are taken as they are in nearly every tile"""
    page, queries = 16, 26
    cache = filled(20, 1, page, d, 4)
    table = torch.arange(20)[None]
    seen = torch.tensor([[320 - (queries - 1 - i) for i in range(queries)]])
    q = (torch.randn(1, queries, 3, d, generator=torch.Generator().manual_seed(1)) * size).to(KIND[kind])
    got, lse = run(q, cache, table, seen, 0.09)
    check_far(kind, got, lse, q, cache, table, seen, 0.09, page)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("queries", [1, 40])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_a_first_token_above_the_rest(kind, queries, d):
    """A token some 18 above all others, as first tokens often are: every tile after it has weights far below the largest"""
    page, length = 16, 400
    cache = filled(25, 1, page, d, 6)
    g = torch.Generator().manual_seed(2)
    table = torch.randperm(25, generator=g)[None]
    q = torch.randn(1, queries, 2, d, generator=g)
    q[..., 0] = q[..., 0].abs() + 1
    block = cache[int(table[0, 0]), 0]
    block[:d // 2] = 0
    block[0] = 0x7                                     # the first token's key: one channel, of 12 times its scale
    block[page * d:page * d + 2] = np.frombuffer(np.float16(1.5 * math.sqrt(d)).tobytes(), np.uint8)
    seen = torch.tensor([[length]])
    got, lse = run(q.to(KIND[kind]), cache, table, seen, 1 / math.sqrt(d))
    check(kind, got, lse, q.to(KIND[kind]), cache, table, seen, 1 / math.sqrt(d), 0, page)
