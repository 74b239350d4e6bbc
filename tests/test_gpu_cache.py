"""The 4-bit cache: what appending leaves in it, byte by byte, and reading it back."""
import numpy as np
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, UNITS, half_step, held, rotated, token_of_block, values_of, view

pytestmark = pytest.mark.gpu


def made(lead, heads, d, kind, seed=0, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*lead, heads, d, generator=g) * size).to(KIND[kind])


def new_cache(pages, heads, page, d, fill=0xa5):
    return torch.full((pages, heads, ocn.cache_block_bytes(page, d)), fill, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d,page,heads,lead", [(64, 16, 3, (7,)), (128, 16, 1, (1,)), (128, 48, 8, (2, 19)), (256, 32, 2, (33,)),
                                               (64, 64, 4, (3, 50)), (128, 128, 2, (1, 300))])
def test_append_without_rotation(d, page, heads, lead, kind):
    k, v = made(lead, heads, d, kind), made(lead, heads, d, kind, 1, 30.0)
    n = int(np.prod(lead))
    pages = -(-n // page) + 2
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(3))[:n].view(lead)
    cache = new_cache(pages, heads, page, d)
    before = cache.clone()
    ocn.cache_append(view(k.cuda()), view(v.cuda()), view(slots.cuda()), view(cache))
    got = values_of(cache.cpu().numpy(), page, d)
    flat = slots.reshape(-1).numpy()
    for x, have in zip((k, v), got):
        want = held(x.double().numpy()).reshape(n, heads, d)
        assert np.array_equal(have[flat // page, :, flat % page], want)
    one = token_of_block(cache[flat[0] // page, heads - 1].cpu().numpy(), page, d, flat[0] % page)     # the layout, place by place
    assert np.array_equal(one[0], got[0][flat[0] // page, heads - 1, flat[0] % page])
    assert np.array_equal(one[1], got[1][flat[0] // page, heads - 1, flat[0] % page])
    # nothing else was written: the tokens that were not named hold what they held
    old = values_of(before.cpu().numpy(), page, d)
    rest = np.setdiff1d(np.arange(pages * page), flat)
    for a, b in zip(got, old):
        assert np.array_equal(a[rest // page, :, rest % page], b[rest // page, :, rest % page])
    # reading back: values are exact in half and float, rounded once to bfloat16
    out = [torch.zeros_like(t).cuda() for t in (k, v)]
    ocn.cache_read(view(cache), view(slots.to(torch.int32).cuda()), view(out[0]), view(out[1]))
    for x, y in zip((k, v), out):
        assert torch.equal(y.cpu(), torch.from_numpy(held(x.double().numpy())).to(KIND[kind]))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d,r,inter", [(64, 64, False), (128, 128, False), (128, 32, True), (256, 200, False), (64, 10, False), (128, 24, False)])
def test_append_rotates_keys(d, r, inter, kind):
    lead, heads, page = (3, 21), 2, 16
    k, v = made(lead, heads, d, kind), made(lead, heads, d, kind, 1)
    pos = torch.randint(0, 100000, lead, generator=torch.Generator().manual_seed(1))
    freq = torch.tensor(ocn.rotary_frequencies(r)[0], dtype=torch.float64)
    rot = ocn.Rotation(view(pos.cuda()), view(freq.cuda()), r, "interleaved" if inter else "half", 1.1)
    slots = torch.arange(63).view(lead)
    cache = new_cache(4, heads, page, d)
    # the keys and values side by side in one buffer
    both = torch.cat([k, v], -2).cuda()
    ocn.cache_append(view(both[:, :, :heads]), view(both[:, :, heads:]), view(slots.cuda()), view(cache), rotation=rot)
    have_k, have_v = (x.transpose(0, 2, 1, 3).reshape(-1, heads, d)[:63] for x in values_of(cache.cpu().numpy(), page, d))
    assert np.array_equal(have_v, held(v.double().numpy()).reshape(63, heads, d))
    want, size = (x.numpy().reshape(63, heads, d) for x in rotated(k.double(), pos, freq, r, inter, 1.1))
    err = 5 * F32 * size                                  # of the rotated channel in single precision
    group = lambda x: x.reshape(63, heads, d // 32, 32)  # noqa: E731
    scales = cache[:, :, page * d:page * d + page * d // 16].cpu().contiguous().numpy().view(np.float16)
    scales = scales.reshape(4, heads, d // 32, page).transpose(0, 3, 1, 2).reshape(-1, heads, d // 32)[:63].astype(np.float64)
    top = np.abs(group(want)).max(-1)
    # nine bits: half a step is 2^-9 of the value, and the largest channel has an error itself
    assert (np.abs(scales * 12 - top) <= top * (2.0 ** -9 + 2 * F32) + group(err).max(-1)).all()
    # each value is the nearest one, or as near to within the channel's error
    grid = np.array([s * u for u in UNITS for s in (-1, 1)]) * scales[..., None, None]
    nearest = np.abs(group(want)[..., None] - grid).min(-1)
    assert (np.abs(group(have_k) - group(want)) <= nearest * (1 + 2.0 ** -20) + 2 * group(err) + 2 * F32 * np.abs(group(want))).all()


def test_slots_outside_are_left_out():
    d, page, heads = 128, 16, 2
    k, v = made((6,), heads, d, "half"), made((6,), heads, d, "half", 1)
    slots = torch.tensor([3, -1, 32, 5, 2 ** 40, -2 ** 40])
    cache = new_cache(2, heads, page, d)
    ocn.cache_append(view(k.cuda()), view(v.cuda()), view(slots.cuda()), view(cache))
    got = values_of(cache.cpu().numpy(), page, d)
    old = values_of(new_cache(2, heads, page, d).cpu().numpy(), page, d)
    want = held(k.double().numpy())
    for place in range(32):
        t = {3: 0, 5: 3}.get(place)
        expect = old[0][place // page, :, place % page] if t is None else want[t]
        assert np.array_equal(got[0][place // page, :, place % page], expect)
    out = torch.full((6, heads, d), 9.0, dtype=torch.float16, device="cuda")
    ocn.cache_read(view(cache), view(slots.cuda()), view(out), None)
    assert (out[[1, 2, 4, 5]] == 9).all() and torch.equal(out[[0, 3]].cpu(), torch.from_numpy(want[[0, 3]]).half())


def test_values_at_the_ends():
    d, page = 64, 16
    k = torch.zeros(8, 1, d)
    k[0, 0, :32] = 1e30                                   # saturates
    k[0, 0, 33] = -7e4
    k[1, 0, 3] = float("nan")
    k[2, 0, 40] = float("-inf")
    k[3, 0, 1] = 1e-12                                    # a scale that underflows to zero
    k[4, 0, :3] = torch.tensor([2.0 ** -24, -(2.0 ** -23), 12 * 2.0 ** -24])
    k[5, 0, :8] = torch.tensor([12.0, 0.5, 1.5, 2.5, 3.5, 5.0, 7.0, 10.0])      # ties
    k[6, 0, :8] = -torch.tensor([12.0, 0.5, 1.5, 2.5, 3.5, 5.0, 7.0, 10.0])
    k[7, 0] = -0.0
    v = k.flip(0).contiguous()
    cache = new_cache(1, 1, page, d)
    ocn.cache_append(view(k.cuda()), view(v.cuda()), view(torch.arange(8).cuda()), view(cache))
    out = [torch.zeros(8, 1, d, device="cuda") for _ in range(2)]
    ocn.cache_read(view(cache), view(torch.arange(8).cuda()), view(out[0]), view(out[1]))
    a, b = (x.cpu() for x in out)
    assert torch.equal(a.nan_to_num(5.5), b.flip(0).nan_to_num(5.5))
    a = a[:, 0]
    assert (a[0, :32] == 65472).all() and a[0, 33] == -65472 and (a[0, 34:] == 0).all()
    assert a[1, :32].isnan().all() and (a[1, 32:] == 0).all() and a[2, 32:].isnan().all() and (a[2, :32] == 0).all()
    assert (a[3] == 0).all()
    assert torch.equal(a[4, :4], torch.tensor([2.0 ** -24, -(2.0 ** -23), 12 * 2.0 ** -24, 0.0]))
    assert a[5, :8].tolist() == [12, 0, 2, 2, 4, 4, 8, 8] and a[6, :8].tolist() == [-12, 0, -2, -2, -4, -4, -8, -8]
    assert (a[7] == 0).all() and a[7].signbit().all()


def test_strided_operands_and_cache():
    d, page, heads, n = 128, 32, 3, 21
    kind = "bfloat16"
    k, v = made((n,), heads, d, kind), made((n,), heads, d, kind, 1)
    wide = torch.full((5, heads + 1, ocn.cache_block_bytes(page, d) + 64), 0x5a, dtype=torch.uint8, device="cuda")
    cache = wide[1:, 1:, :ocn.cache_block_bytes(page, d)]
    slots = torch.arange(n).cuda()
    a = torch.zeros(n, heads, d, 2, dtype=KIND[kind], device="cuda")[..., 1]          # channels apart
    a.copy_(k)
    b = torch.zeros(heads, n, d, dtype=KIND[kind], device="cuda").transpose(0, 1)     # heads first
    b.copy_(v)
    ocn.cache_append(view(a), view(b), view(slots), view(cache))
    out = [torch.zeros(n, heads, d, dtype=KIND[kind], device="cuda") for _ in range(2)]
    ocn.cache_read(view(cache), view(slots), view(out[0]), view(out[1]))
    for x, y in zip((k, v), out):
        assert torch.equal(y.cpu(), torch.from_numpy(held(x.double().numpy())).to(KIND[kind]))
    assert (wide[0] == 0x5a).all() and (wide[:, 0] == 0x5a).all() and (wide[:, :, ocn.cache_block_bytes(page, d):] == 0x5a).all()
    assert half_step(kind) == 2.0 ** -8
