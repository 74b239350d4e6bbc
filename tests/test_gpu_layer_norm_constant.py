"""The layer norm and its gradient for rows that are constant or nearly so, far from zero.

Bounds.  u = 2^-24 is half a step of single precision.  A constant row is its own mean: deviations, and what they add to gradients, are zeros, and results are those of the bias.
Nearly constant ones in single precision, with W channels: the sum, in 64 bits, is off by W 2^-53 of mean|x|; what the mean is more than its rounding to single precision, half a step of it at most, is itself
rounded, u of it; a deviation is rounded twice more, and the variance a sum of W squares over 16 channels of a lane, 6 exchanges and 16 wavefronts, which with the square root, r and its product make
64 u at most."""
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, rounding, view
from test_gpu_heads import check

pytestmark = pytest.mark.gpu

WIDTHS = [3, 64, 100, 405, 821, 942, 1500, 3001, 5003, 6000, 10000, 16383]
# constants with all the bits that their type has, and others
CONSTANTS = {"float": [152840384.0, 16066.638, 197021.7, -1e9, 3.3333333e6, 1e30, 1234.5678], "half": [60000.0, 1000.5, -2047.0, 0.33325], "bfloat16": [1e6, -1.9921875, 255.0, 3e30]}


def run(x, g, w, b, eps):
    out, gin, gw, gb = torch.full_like(x, 7.0).cuda(), torch.full_like(x, 7.0).cuda(), torch.full((x.shape[-1],), 7.0).cuda(), torch.full((x.shape[-1],), 7.0).cuda()
    xs, ws = view(x.cuda()), view(w.cuda())
    ocn.layer_norm(xs, ws, view(b.cuda()), view(out), eps=eps)
    ocn.layer_norm_grad(view(g.cuda()), xs, ws, view(gin), view(gw), view(gb), eps=eps)
    return out, gin, gw, gb


def random(*sizes, seed):
    return torch.randn(*sizes, generator=torch.Generator().manual_seed(seed))


def grad_of(g, w, u, r):
    """The gradient of x for unit rows u, with what it loses in single precision where u and r are right"""
    h = g.double() * w.double()
    mean_h, mean_hu = h.mean(-1, keepdim=True), (h * u).mean(-1, keepdim=True)
    size = h.abs() + h.abs().mean(-1, keepdim=True) + u.abs() * (h * u).abs().mean(-1, keepdim=True)
    return r * (h - mean_h - u * mean_hu), r * 64 * F32 * size, h


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_constant_rows(kind, eps):
    for width in WIDTHS:
        x = torch.tensor(CONSTANTS[kind]).to(KIND[kind])[:, None].repeat(1, width)
        g, w, b = random(len(x), width, seed=1).to(KIND[kind]), 1 + random(width, seed=2) / 4, random(width, seed=3)
        out, gin, gw, gb = run(x, g, w, b, eps)
        assert torch.equal(out.cpu(), b.to(KIND[kind]).expand_as(x)), width
        if eps > 1e-10:      # (and in half precision results stay in range)
            want, bound, _ = grad_of(g, w, torch.zeros(x.shape, dtype=torch.float64), eps ** -0.5)
            check(gin, want, rounding(kind, want) + bound)
        assert (gw == 0).all(), width
        want = g.double().sum(0)
        check(gb, want, rounding("float", want) + len(x) * F32 * g.double().abs().sum(0))


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_nearly_constant_rows(eps):
    """One to three values of single precision that follow each other"""
    for width in WIDTHS:
        c = torch.tensor([x for x in CONSTANTS["float"] if abs(x) < 1e20])[:, None]
        step = 2.0 ** (torch.floor(torch.log2(c.abs())) - 23)
        x = c + step * torch.randint(-1, 2, (len(c), width), generator=torch.Generator().manual_seed(width))
        assert ((x.double() - c.double()).abs() <= 2 * step).all()
        g, w, b = random(len(x), width, seed=1), 1 + random(width, seed=2) / 4, random(width, seed=3)
        out, gin, gw, gb = run(x, g, w, b, eps)
        xd = x.double()
        m = xd[:, :1] + (xd - xd[:, :1]).mean(-1, keepdim=True)
        r = 1 / ((xd - m).square().mean(-1, keepdim=True) + float(torch.tensor(eps))).sqrt()
        u = (xd - m) * r
        mean_off = (width + 1) * 2.0 ** -53 * xd.abs().mean(-1, keepdim=True) + F32 * F32 * m.abs()
        off = r * mean_off * 2 + u.abs() * (64 * F32 + 2 * (r * mean_off))
        want = u * w.double() + b.double()
        check(out, want, rounding("float", want) + off * w.double().abs() + 2 * F32 * want.abs())
        want, bound, h = grad_of(g, w, u, r)
        bound = bound + r * (off * (h * u).abs().mean(-1, keepdim=True) + u.abs() * (h.abs() * off).mean(-1, keepdim=True)) + want.abs() * (64 * F32 + 2 * r * mean_off)
        check(gin, want, rounding("float", want) + bound)
        want = (g.double() * u).sum(0)
        check(gw, want, rounding("float", want) + (g.double().abs() * (off + (len(x) + 2) * F32 * u.abs())).sum(0))


def test_other_rows_are_as_they_were():
    """NaN and infinities reach their own rows, whole"""
    for width in (100, 942, 5003):
        for kind in KIND:
            x = torch.full((5, width), 1000.0).to(KIND[kind])
            x[1, 3], x[2, 50], x[3, 99] = float("nan"), float("inf"), -float("inf")
            out, gin, gw, _ = run(x, torch.ones_like(x), torch.ones(width), torch.zeros(width), 1e-5)
            for t in (out, gin):
                assert t[1:4].isnan().all() and t[[0, 4]].isfinite().all()
            assert gw.isnan().all()
