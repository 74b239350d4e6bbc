"""Rotations by positions on several axes, in every call that takes a rotation, against 64-bit forms.  Bounds as for one axis: the angle is a sum in double precision."""
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, normed, rounding, values_of, view
from test_gpu_heads import check, gradients, made, spread

pytestmark = pytest.mark.gpu

# lead, heads, channels, pairs of each axis, order, interleaved
SHAPES = [((1,), 4, 64, (12, 10, 10), "row", False), ((3, 7), 5, 128, (16, 24, 24), "row", False), ((2, 33), 8, 128, (22, 21, 21), "turn", False),
          ((65,), 3, 96, (8, 8, 8), "turn", True), ((11,), 2, 80, (20, 20), "row", False), ((9,), 2, 33, (3, 7), "turn", False), ((700,), 3, 256, (64, 0, 32, 32), "turn", True),
          ((5,), 2, 64, (32,), "row", False), ((4, 5), 2, 512, (100, 78, 78), "row", False)]


def rotation_of(shape, start=0, wide=False, magnitude=1.0):
    lead, _, _, pairs, order, inter = shape
    g = torch.Generator().manual_seed(sum(lead))
    pos = (start + torch.randint(0, 5000, (len(pairs),) + lead, generator=g)).to(torch.int64 if wide else torch.int32)
    n = sum(pairs)
    table = torch.tensor(ocn.rotary_axes(pairs, ocn.rotary_frequencies(2 * n)[0], order), dtype=torch.float64)
    dev = pos.cuda(), table.cuda()
    return pos, table, ocn.Rotation(view(dev[0]), view(dev[1]), 2 * n, "interleaved" if inter else "half", magnitude)


def turned(x, pos, table, inter, magnitude=1.0, back=False):
    """As heads_ref.rotated, by the sum over the axes"""
    angle = (pos.double()[..., None] * table.view(table.shape[0], *[1] * (pos.dim() - 1), -1)).sum(0)
    r = 2 * table.shape[1]
    angle = angle.expand(*x.shape[:-2], r // 2)[..., None, :]
    c, s = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if back else 1)
    a, b = (slice(0, r, 2), slice(1, r, 2)) if inter else (slice(0, r // 2), slice(r // 2, r))
    out, size = x.clone(), x.abs()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    return out, size


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotary(shape, kind):
    lead, heads, d, _, _, inter = shape
    x = made(lead, heads, d, kind)
    for back, how in ((False, ""), (True, "packed"), (False, "off by one")):
        pos, table, rot = rotation_of(shape, -3 if back else 1 << 20, wide=back, magnitude=0.75 if back else 1.0)
        out = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
        ocn.rotary(view(spread(x.cuda(), how)), rot, view(out), inverse=back)
        want, size = turned(x.double(), pos, table, inter, rot.magnitude, back)
        check(out, want, rounding(kind, want) + 5 * F32 * size)


def test_equal_positions_are_one_axis():
    """A text's tokens have the same position on all axes: the bits of a rotation with one"""
    x = made((50,), 3, 128, "bfloat16").cuda()
    at = torch.arange(777, 827, dtype=torch.int32).cuda()
    f = ocn.rotary_frequencies(128)[0]
    one, many = torch.zeros_like(x), torch.zeros_like(x)
    ocn.rotary(view(x), ocn.Rotation(view(at), view(torch.tensor(f, dtype=torch.float64).cuda()), 128), view(one))
    for order in ("row", "turn"):
        table = torch.tensor(ocn.rotary_axes((16, 24, 24), f, order), dtype=torch.float64).cuda()
        ocn.rotary(view(x), ocn.Rotation(view(at.expand(3, 50)), view(table), 128), view(many))
        assert torch.equal(one, many)


def test_positions_broadcast_and_tables_of_any_layout():
    """Sequences that share positions, frequencies of pairs that turn by all axes, a transposed table and reversed axes"""
    x = made((4, 6), 2, 64, "float")
    table = torch.rand(3, 32, dtype=torch.float64, generator=torch.Generator().manual_seed(3))
    dev = table.t().contiguous().cuda().t()
    for pos in (torch.arange(18).view(3, 6), torch.arange(3).view(3, 1), torch.arange(12).view(3, 4, 1), torch.tensor([7, -9, 100000])):
        at = pos.cuda()
        out = torch.zeros_like(x).cuda()
        ocn.rotary(view(x.cuda()), ocn.Rotation(view(at), view(dev), 64), view(out))
        want, size = turned(x.double(), pos, table, False)
        check(out, want, rounding("float", want) + 5 * F32 * size)
        v, t = view(at), view(dev)
        back = [ocn.Tensor(w.base + 2 * w.strides[0], w.dtype, w.sizes, (-w.strides[0],) + w.strides[1:], 0, 0, k) for w, k in ((v, at), (t, dev))]
        again = torch.zeros_like(x).cuda()
        ocn.rotary(view(x.cuda()), ocn.Rotation(back[0], back[1], 64), view(again))
        check(again, want, rounding("float", want) + 5 * F32 * size)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_and_gradient(shape, kind):
    lead, heads, d, _, _, inter = shape
    pos, table, rot = rotation_of(shape, 400)
    q, k, gq, gk = (made(lead, n, d, kind, s) for n, s in ((heads, 0), (2, 1), (heads, 2), (2, 3)))
    w = [1 + made((), 1, d, "float", s)[0] / 4 for s in (4, 5)]
    out = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") for t in (q, k)]
    gin = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") for t in (q, k)]
    gw = [torch.zeros(d, device="cuda") for _ in range(2)]
    vw = [view(t.cuda()) for t in w]
    ocn.norm_rotary(view(q.cuda()), vw[0], view(out[0]), view(k.cuda()), vw[1], view(out[1]), eps=1e-5, rotation=rot)
    ocn.norm_rotary_grad(view(gq.cuda()), view(q.cuda()), vw[0], view(gin[0]), view(gw[0]), view(gk.cuda()), view(k.cuda()), vw[1], view(gin[1]), view(gw[1]),
                         eps=1e-5, rotation=rot)
    for i, (x, g) in enumerate(((q, gq), (k, gk))):
        want, size = turned(normed(x.double(), w[i].double(), 1e-5), pos, table, inter)
        check(out[i], want, rounding(kind, want) + (d / 2 + 12) * F32 * size)
        h, h_size = turned(g.double(), pos, table, inter, back=True)
        gx, _, gweight, _, _ = gradients(x.double(), h, w[i].double(), 1e-5, None, None, 0, False)
        _, gx_size, _, gw_size, _ = gradients(x.double(), h_size, w[i].double(), 1e-5, None, None, 0, False)
        check(gin[i], gx, rounding(kind, gx) + (2 * d + 24) * F32 * gx_size)
        check(gw[i], gweight, rounding("float", gweight) + (x.numel() // d + d / 2 + 24) * F32 * gw_size)


def test_appending_to_the_cache():
    """Keys rotated on the way hold the same codes as keys rotated before, where that rounds nothing"""
    shape = ((2, 20), 3, 64, (12, 10, 10), "row", False)
    pos, table, rot = rotation_of(shape)
    k, v = made((2, 20), 3, 64, "float").cuda(), made((2, 20), 3, 64, "float", 1).cuda()
    slots = torch.arange(40, dtype=torch.int32).view(2, 20).cuda()
    caches = [torch.zeros(3, 3, ocn.cache_block_bytes(16, 64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    ocn.cache_append(view(k), view(v), view(slots), view(caches[0]), rotation=rot)
    ocn.rotary(view(k), rot, view(k))
    ocn.cache_append(view(k), view(v), view(slots), view(caches[1]))
    assert torch.equal(caches[0], caches[1]) and values_of(caches[0].cpu().numpy(), 16, 64)[0].any()
