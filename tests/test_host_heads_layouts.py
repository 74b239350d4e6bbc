"""Queries, keys and values in one buffer: which layouts the operators over heads take as not sharing bytes (no GPU)."""
import itertools
import random

import pytest

import paper_1810_08723_amd as ocn
from test_host_heads import T, code, rot

W = T("float", (64,), base=4)


def taken(q, k, w=W):
    """Whether queries and keys normed in place get past the checks of sharing: positions that fit no call are refused after those"""
    got = code(ocn.norm_rotary, q, w, q, k, w, k, rotation=rot(2, pos=T("int32", (1000,), base=8)))
    assert got in ("SHAPE", "ALIAS", "OVERLAP_OUT")
    return got == "SHAPE"


def parts(order, batch, tokens, counts, d, size=2):
    """Views [batch, tokens, heads, channels] of one buffer of sum(counts) heads; `order`: its dimensions, slowest first"""
    sizes = {"b": batch, "t": tokens, "h": sum(counts), "d": d}
    strides, acc = {}, size
    for n in reversed(order):
        strides[n] = acc
        acc *= sizes[n]
    at, out = 0, []
    for c in counts:
        out.append(((batch, tokens, c, d), tuple(strides[n] for n in "bthd"), at * strides["h"]))
        at += c
    return out


def view(part, kind="half", base=0):
    sizes, strides, offset = part
    return T(kind, sizes, strides, base=base, offset=offset)


@pytest.mark.parametrize("order", ["".join(p) for p in itertools.permutations("bthd")])
@pytest.mark.parametrize("counts", [(8, 2, 2), (1, 1, 1), (4, 1, 1), (3, 5, 5)])
@pytest.mark.parametrize("batch,tokens", [(3, 5), (1, 5), (3, 1), (1, 1)])
def test_one_buffer_in_any_order(order, counts, batch, tokens):
    q, k, v = (view(p) for p in parts(order, batch, tokens, counts, 64))
    assert taken(q, k)
    cache = T("uint8", (0, counts[1], ocn.cache_block_bytes(16, 64)), base=3)     # (of no pages: nothing is launched)
    ocn.cache_read(cache, T("int64", (batch, tokens), base=2), k, v, stream=0)


def test_heads_that_meet():
    for order in ("bthd", "bhtd", "hbtd", "tbhd"):
        q, k, _ = parts(order, 3, 5, (8, 2, 2), 64)
        for shift in (-1, -2, -7):          # heads that are queries' as well
            moved = (k[0], k[1], k[2] + shift * k[1][2])
            assert not taken(view(q), view(moved))
        if order == "bhtd":                 # one token further on: the last head's last token is the next sequence's first
            moved = (k[0], k[1], k[2] + 3 * k[1][1] + 2 * k[1][2])
            assert not taken(view(q), view(moved))


def elements(part):
    sizes, strides, offset = part
    return {offset + sum(i * s for i, s in zip(at, strides)) for at in itertools.product(*map(range, sizes))}


def test_views_that_share_are_refused():
    """Against the bytes themselves, for small views of any strides: what shares is refused"""
    rng = random.Random(5)
    shared = passed = 0
    for _ in range(4000):
        lead = rng.randint(1, 2)
        sizes = [rng.randint(1, 3) for _ in range(lead)]
        strides = [2 * rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 24, 48, -4, -8, -24)) for _ in range(lead)]
        two = []
        for _ in range(2):
            more = [2 * rng.choice((1, 2, 3, 4, 6, 8, 12, 16, 24, -2, -4, -8)) for _ in range(2)]
            mine = strides if rng.random() < 0.8 else [s * 2 for s in strides]
            two.append((tuple(sizes + [rng.randint(1, 3), 2]), tuple(mine + more), 1000 + 2 * rng.randint(0, 40)))
        a, b = two
        if any(len(elements(p)) < p[0][-1] * p[0][-2] * len(list(itertools.product(*map(range, p[0][:-2])))) for p in two):
            continue
        got = taken(view(a), view(b), T("float", (2,), base=4))
        if elements(a) & elements(b):
            shared += 1
            assert not got, (a, b)
        else:
            passed += got
    assert shared > 200 and passed > 200
