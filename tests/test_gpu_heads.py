"""Rotary positions and norms of heads against 64-bit forms.  Bounds: one rounding of the result to its type (half a step), plus
what single precision loses before it: a pair's rotation is two products, a sum and two rounded factors (4 half steps of
|a| + |b|); a norm has a sum of D squares, and a handful of roundings."""
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, half_step, normed, rotated, rounding, view

pytestmark = pytest.mark.gpu

# lead, heads, channels, rotary_dim, interleaved
SHAPES = [((1,), 1, 64, 64, False), ((1, 1), 32, 128, 128, False), ((3, 7), 5, 128, 128, False), ((2, 33), 8, 128, 64, True),
          ((65,), 3, 96, 48, False), ((5,), 9, 80, 40, False), ((2, 3), 2, 48, 24, False), ((4, 5), 7, 50, 50, False), ((9,), 2, 33, 20, False),
          ((11,), 3, 7, 2, True), ((300,), 40, 128, 128, False), ((17,), 6, 256, 256, True), ((6,), 2, 512, 512, False), ((2, 2, 2), 3, 128, 16, False),
          ((0,), 4, 64, 64, False), ((4,), 0, 64, 64, False), ((2, 3, 1, 4, 2), 1, 64, 32, True), ((700,), 1, 64, 64, False)]


def spread(t, how):
    """The same values in another layout"""
    if how == "packed":        # the middle heads of wider rows
        wide = torch.randn(*t.shape[:-2], t.shape[-2] + 5, t.shape[-1], device=t.device).to(t.dtype)
        out = wide[..., 2:2 + t.shape[-2], :]
    elif how == "channels":    # channels apart
        out = torch.zeros(*t.shape, 3, dtype=t.dtype, device=t.device)[..., 1]
    elif how == "heads first":
        out = torch.zeros(t.shape[-2], *t.shape[:-2], t.shape[-1], dtype=t.dtype, device=t.device).movedim(0, -2)
    elif how == "off by one":  # rows that start between vectors
        flat = torch.zeros(t.numel() + 1, dtype=t.dtype, device=t.device)
        out = flat[1:].view(t.shape)
    else:
        return t
    out.copy_(t)
    return out


def made(lead, heads, d, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(*lead, heads, d, generator=g).to(KIND[kind])


def rotation_of(lead, rotary_dim, interleaved, start, wide=False, magnitude=1.0, stretch="none"):
    g = torch.Generator().manual_seed(len(lead))
    pos = (start + torch.randint(0, 1000, lead or (1,), generator=g)).to(torch.int64 if wide else torch.int32)
    f, _ = ocn.rotary_frequencies(rotary_dim, 10000.0, stretch, 4.0)
    freq = torch.tensor(f, dtype=torch.float64)
    dev = pos.cuda(), freq.cuda()
    return pos, freq, ocn.Rotation(view(dev[0]), view(dev[1]), rotary_dim, "interleaved" if interleaved else "half", magnitude)


def check(got, want, bound):
    got = got.double().cpu()
    assert got.shape == want.shape
    worst = ((got - want).abs() - bound).max().item() if want.numel() else 0.0
    assert worst <= 0, worst


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotary(shape, kind):
    lead, heads, d, r, inter = shape
    x = made(lead, heads, d, kind)
    for back in (False, True):
        pos, freq, rot = rotation_of(lead, r, inter, 0 if back else 1 << 20, wide=back, magnitude=1.25 if back else 1.0, stretch="linear")
        out = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
        ocn.rotary(view(x.cuda()), rot, view(out), inverse=back)
        want, size = rotated(x.double(), pos, freq, r, inter, rot.magnitude, back)
        check(out, want, rounding(kind, want) + 5 * F32 * size)


@pytest.mark.parametrize("how", ["packed", "channels", "heads first", "off by one"])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[4], SHAPES[5], SHAPES[7]], ids=str)
def test_rotary_layouts(shape, how):
    lead, heads, d, r, inter = shape
    for kind in KIND:
        x = made(lead, heads, d, kind)
        pos, freq, rot = rotation_of(lead, r, inter, 31)
        want, size = rotated(x.double(), pos, freq, r, inter)
        a = spread(x.cuda(), how)
        out = spread(torch.zeros_like(x).cuda(), how)
        ocn.rotary(view(a), rot, view(out))
        check(out, want, rounding(kind, want) + 5 * F32 * size)
        ocn.rotary(view(a), rot, view(a))                      # in place
        assert torch.equal(a, out)
        other = torch.zeros_like(x).cuda()
        ocn.rotary(view(out), rot, view(other), inverse=True)  # and back: a rounding more
        check(other, x.double(), 3 * half_step(kind) * (want.abs() + size) + 16 * F32 * size)


def test_positions_broadcast_and_channels_outside_stay():
    x = made((3, 6), 4, 64, "float")
    x[..., 40:] = float("inf")
    x[1, :, :, 50] = float("nan")
    freq = torch.tensor(ocn.rotary_frequencies(32)[0], dtype=torch.float64)
    for pos in (torch.arange(6), torch.tensor([5]), torch.arange(3)[:, None], torch.tensor(9)):
        rot = ocn.Rotation(view(pos.cuda()), view(freq.cuda()), 32)
        out = torch.zeros_like(x).cuda()
        ocn.rotary(view(x.cuda()), rot, view(out))
        want, size = rotated(x.double(), pos, freq, 32)
        assert torch.equal(out[..., 32:].cpu().nan_to_num(1.5), x[..., 32:].nan_to_num(1.5))
        check(out[..., :32], want[..., :32], rounding("float", want[..., :32]) + 5 * F32 * size[..., :32])


def test_far_positions():
    x = made((4,), 2, 64, "float")
    pos = torch.tensor([2 ** 31 - 1, 2 ** 30 + 12345, -(2 ** 31), 10 ** 9 + 7])
    freq = torch.tensor(ocn.rotary_frequencies(64)[0], dtype=torch.float64)
    rot = ocn.Rotation(view(pos.cuda()), view(freq.cuda()), 64)
    out = torch.zeros_like(x).cuda()
    ocn.rotary(view(x.cuda()), rot, view(out))
    want, size = rotated(x.double(), pos, freq, 64)
    # (the angle itself is rounded once: half a step of 2^31 in 64 bits is 2^-23)
    check(out, want, rounding("float", want) + 5 * F32 * size + 2.0 ** -22 * size)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_rotary(shape, kind):
    lead, heads, d, r, inter = shape
    pos, freq, rot = rotation_of(lead, r, inter, 4000)
    q, k = made(lead, heads, d, kind), made(lead, 2, d, kind, 1)
    for wkind, turn in (("float", True), (kind, True), (None, True), (kind, False)):
        w = [None if wkind is None else 1 + made((), 1, d, wkind, s)[0] / 4 for s in (3, 4)]
        out = [torch.full(t.shape, 7.0, dtype=t.dtype, device="cuda") for t in (q, k)]
        args = [None if x is None else view(x.cuda()) for x in w]
        ocn.norm_rotary(view(q.cuda()), args[0], view(out[0]), view(k.cuda()), args[1], view(out[1]), eps=1e-5, rotation=rot if turn else None)
        for x, weight, got in zip((q, k), w, out):
            y = normed(x.double(), 1.0 if weight is None else weight.double(), 1e-5)
            want, size = rotated(y, pos, freq, r, inter) if turn else (y, y.abs())
            check(got, want, rounding(kind, want) + (d / 2 + 12) * F32 * size)


def test_norm_in_place_in_a_packed_buffer():
    qkv = made((3, 5), 12, 128, "bfloat16").cuda()
    pos, freq, rot = rotation_of((3, 5), 128, False, 0)
    want = [torch.zeros(3, 5, n, 128, dtype=torch.bfloat16, device="cuda") for n in (8, 2)]
    q, k = qkv[:, :, :8], qkv[:, :, 8:10]
    rest = qkv[:, :, 10:].clone()
    ocn.norm_rotary(view(q), None, view(want[0]), view(k), None, view(want[1]), rotation=rot)
    ocn.norm_rotary(view(q), None, view(q), view(k), None, view(k), rotation=rot)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(qkv[:, :, 10:], rest)


def gradients(x, g, w, eps, pos, freq, r, inter):
    """Formula's gradients in 64 bits, and the sizes that bound their errors"""
    h, size = rotated(g, pos, freq, r, inter, back=True) if pos is not None else (g, g.abs())
    d = x.shape[-1]
    rr = 1 / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    u = x * rr
    hw = h * w
    gx = rr * (hw - u * (hw * u).mean(-1, keepdim=True))
    gx_size = rr * ((size * w.abs()) + u.abs() * (size * w.abs() * u.abs()).mean(-1, keepdim=True))
    flat = tuple(range(x.dim() - 1))
    return gx, gx_size, (h * u).sum(flat), (size * u.abs()).sum(flat), d


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_norm_rotary_grad(shape, kind):
    lead, heads, d, r, inter = shape
    pos, freq, rot = rotation_of(lead, r, inter, 77)
    xs, gs = [made(lead, n, d, kind, n) for n in (heads, 2)], [made(lead, n, d, kind, n + 9) for n in (heads, 2)]
    for wkind, turn in (("float", True), (kind, False)):
        ws = [1 + made((), 1, d, wkind, s)[0] / 4 for s in (3, 4)]
        gin = [torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda") for x in xs]
        gw = [torch.full((d,), 7.0, dtype=KIND[wkind], device="cuda") for _ in xs]
        v = [[view(t.cuda()) for t in ts] for ts in (gs, xs, ws)]
        ocn.norm_rotary_grad(v[0][0], v[1][0], v[2][0], view(gin[0]), view(gw[0]), v[0][1], v[1][1], v[2][1], view(gin[1]), view(gw[1]),
                             eps=1e-5, rotation=rot if turn else None)
        for i in range(2):
            gx, gx_size, gweight, gw_size, _ = gradients(xs[i].double(), gs[i].double(), ws[i].double(), 1e-5, pos if turn else None, freq, r, inter)
            check(gin[i], gx, rounding(kind, gx) + (2 * d + 24) * F32 * gx_size)
            rows = xs[i].numel() // max(d, 1)
            check(gw[i], gweight, rounding(wkind, gweight) + (rows + d / 2 + 24) * F32 * gw_size)


def test_gradient_against_differences():
    """The gradient of sum(out * g) by central differences of the forward call in 64 bits"""
    lead, heads, d = (3,), 2, 16
    pos, freq, rot = rotation_of(lead, d, False, 5)
    x, g, w = made(lead, heads, d, "float"), made(lead, heads, d, "float", 2), 1 + made((), 1, d, "float", 3)[0] / 4
    gin, gw = torch.zeros_like(x).cuda(), torch.zeros(d).cuda()
    ocn.norm_rotary_grad(view(g.cuda()), view(x.cuda()), view(w.cuda()), view(gin), view(gw), eps=1e-5, rotation=rot)
    f = lambda x, w: (rotated(normed(x, w, 1e-5), pos, freq, d)[0] * g.double()).sum().item()  # noqa: E731
    step = 1e-6
    for i in range(0, x.numel(), 7):
        e = torch.zeros(x.numel(), dtype=torch.float64)
        e[i] = step
        e = e.view(x.shape)
        slope = (f(x.double() + e, w.double()) - f(x.double() - e, w.double())) / (2 * step)
        assert abs(slope - gin.flatten()[i].item()) < 1e-5
    for i in range(d):
        e = torch.zeros(d, dtype=torch.float64)
        e[i] = step
        slope = (f(x.double(), w.double() + e) - f(x.double(), w.double() - e)) / (2 * step)
        assert abs(slope - gw[i].item()) < 1e-5


def test_gradient_in_place_repeats_and_packed():
    lead, d = (2, 301), 128
    pos, freq, rot = rotation_of(lead, d, False, 5)
    qkv, gy = made(lead, 12, d, "bfloat16").cuda(), made(lead, 10, d, "bfloat16", 4).cuda()
    w = (1 + made((), 1, d, "bfloat16", 3)[0] / 4).cuda()
    q, k, gq, gk = qkv[:, :, :8], qkv[:, :, 8:10], gy[:, :, :8], gy[:, :, 8:]

    def call(tq, tk):
        gw = [torch.zeros(d, device="cuda") for _ in range(2)]
        ocn.norm_rotary_grad(view(gq), view(q), view(w), view(tq), view(gw[0]), view(gk), view(k), view(w), view(tk), view(gw[1]), rotation=rot)
        return gw

    first = [torch.zeros(*lead, n, d, dtype=torch.bfloat16, device="cuda") for n in (8, 2)]
    gw = call(*first)
    again = [torch.zeros_like(t) for t in first]
    assert all(torch.equal(a, b) for a, b in zip(gw, call(*again)))
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    gw2 = call(gq, gk)                                       # in the place of the gradients that come in
    assert torch.equal(gq, first[0]) and torch.equal(gk, first[1]) and all(torch.equal(a, b) for a, b in zip(gw, gw2))


def test_extreme_rows():
    """Zero rows, infinities and NaN stay in their rows"""
    x = made((6,), 1, 64, "float")
    x[0] = 0
    x[2, 0, 5] = float("nan")
    x[4, 0, 9] = float("inf")
    out = torch.zeros_like(x).cuda()
    ocn.norm_rotary(view(x.cuda()), None, view(out), eps=1e-6)
    out = out.cpu()
    assert (out[0] == 0).all() and out[2].isnan().all() and out[[1, 3, 5]].isfinite().all()
    assert out[4, 0, 9].isnan() and (out[4, 0, :9] == 0).all()


def test_many_items_over_a_capped_grid():
    from paper_1810_08723_amd import binding
    x = made((400,), 9, 128, "half")
    pos, freq, rot = rotation_of((400,), 128, False, 5)
    want, got = torch.zeros_like(x).cuda(), torch.zeros_like(x).cuda()
    ocn.norm_rotary(view(x.cuda()), None, view(want), rotation=rot)
    binding.set_max_launch_blocks(3)
    try:
        ocn.norm_rotary(view(x.cuda()), None, view(got), rotation=rot)
        torch.cuda.synchronize()
    finally:
        binding.set_max_launch_blocks(0)
    assert torch.equal(want, got)
