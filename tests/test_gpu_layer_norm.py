"""The layer norm and its gradient against 64-bit forms.

Bounds: one rounding of the result to its type, plus what single precision loses before it.  With W channels and u = (x - m) / s: a sum of W terms over at most 16 channels of
a lane, 6 exchanges and 16 wavefronts is off by at most 40 half steps of the sum of magnitudes, and so are the mean, of mean|x|, and the variance.  For half and bfloat16 the
mean's error is a shift of all deviations; for float it is taken away again, and what is left is that of the deviations."""
import pytest
import torch

import paper_1810_08723_amd as ocn
from heads_ref import F32, KIND, rounding, view
from test_gpu_heads import check, spread

pytestmark = pytest.mark.gpu

# rows of every form: inside a wavefront (1 to 64 lanes, two and four chunks), four wavefronts, sixteen
SHAPES = [((1,), 1), ((5,), 7), ((3, 4), 8), ((700,), 9), ((2, 33), 64), ((1000,), 96), ((4,), 129), ((3,), 512), ((7,), 513), ((65,), 1000), ((5,), 1024), ((9,), 1025),
          ((1030,), 2048), ((3,), 2049), ((2, 3), 4096), ((1, 2), 4097), ((5,), 8192), ((3,), 8200), ((2,), 16383), ((3,), 16384), ((0,), 64), ((4,), 0), ((2, 3, 1, 4, 2), 40)]


def made(lead, width, kind, seed=0, offset=0.0):
    return (torch.randn(*lead, width, generator=torch.Generator().manual_seed(seed)) + offset).to(KIND[kind])


def factors(width, kind, seed, middle):
    return None if kind is None else (middle + made((), width, kind, seed).float() / 4).to(KIND[kind])


def optional(t):
    return None if t is None else view(t.cuda())


def parts(x, eps):
    """u, 1 / s, and how far u may be off in single precision: of shifts of the mean, of the variance, and of its own roundings"""
    w = max(x.shape[-1], 1)
    m = x.mean(-1, keepdim=True)
    r = 1 / ((x - m).square().mean(-1, keepdim=True) + eps).sqrt()
    u = (x - m) * r
    shift = 40 * F32 * x.abs().mean(-1, keepdim=True) * r
    return u, r, shift, w


def bound_of_u(u, r, shift, x, kind):
    if kind == "float":       # (the shift is gone; a deviation is rounded once, and the mean of the deviations is off by 40 half steps of theirs)
        shift = 2 * shift * F32 * 40 + 44 * F32 * u.abs().mean(-1, keepdim=True) + F32 * x.abs() * r * 0
    return shift + u.abs() * (shift ** 2 + 30 * F32) + 2 * F32 * u.abs()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_layer_norm(shape, kind):
    lead, width = shape
    for wkind, bkind, offset, eps in (("float", "float", 0.0, 1e-5), (kind, kind, 3.0, 1e-3), (None, "bfloat16", -1.0, 1e-5), ("half", None, 0.0, 1e-5), (None, None, 0.5, 1e-5)):
        x, w, b = made(lead, width, kind, 1, offset), factors(width, wkind, 2, 1.0), factors(width, bkind, 3, 0.0)
        out = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
        ocn.layer_norm(view(x.cuda()), optional(w), optional(b), view(out), eps=eps)
        xd = x.double()
        u, r, shift, _ = parts(xd, eps)
        wd, bd = (torch.full((), f, dtype=torch.float64) if t is None else t.double() for t, f in ((w, 1.0), (b, 0.0)))
        want = u * wd + bd
        check(out, want, rounding(kind, want) + bound_of_u(u, r, shift, xd, kind) * wd.abs() + F32 * (want.abs() + 1e-30))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_layer_norm_grad(shape, kind):
    lead, width = shape
    for wkind, gkind, offset in (("float", "float", 0.0), (kind, kind, 2.0), (None, "float", 0.0)):
        x, g, w = made(lead, width, kind, 1, offset), made(lead, width, kind, 5), factors(width, wkind, 2, 1.0)
        gin = torch.full(x.shape, 7.0, dtype=x.dtype, device="cuda")
        gweight, gbias = (torch.full((width,), 7.0, dtype=KIND[gkind], device="cuda") for _ in range(2))
        ocn.layer_norm_grad(view(g.cuda()), view(x.cuda()), optional(w), view(gin), None if w is None else view(gweight), view(gbias), eps=1e-5)
        xd, gd, wd = x.double(), g.double(), torch.ones(()).double() if w is None else w.double()
        u, r, shift, n = parts(xd, 1e-5)
        off = bound_of_u(u, r, shift, xd, kind)
        h = gd * wd
        want = r * (h - h.mean(-1, keepdim=True) - u * (h * u).mean(-1, keepdim=True))
        # h is rounded once; its mean is off by 40 half steps of mean|h|, the mean of h u by those of mean|h u| and by u's error in it and beside it
        mean_h, mean_hu = h.abs().mean(-1, keepdim=True), (h * u).abs().mean(-1, keepdim=True)
        size = h.abs() + mean_h + u.abs() * mean_hu
        bound = r * (44 * F32 * size + off * mean_hu + u.abs() * (h.abs() * off).mean(-1, keepdim=True)) + want.abs() * (shift ** 2 + 30 * F32)
        check(gin, want, rounding(kind, want) + bound)
        rows = x.numel() // n
        lead_dims = tuple(range(len(lead)))
        # (a lane's sum over its rows, those of lanes side by side: as many roundings as rows at most; the last sums are in double)
        if w is not None:
            want = (gd * u).sum(lead_dims)
            check(gweight, want, rounding(gkind, want) + (gd.abs() * (off + (rows + 2) * F32 * u.abs())).sum(lead_dims) + 1e-300)
        want = gd.sum(lead_dims)
        check(gbias, want, rounding(gkind, want) + rows * F32 * gd.abs().sum(lead_dims) + 1e-300)


@pytest.mark.parametrize("how", ["channels", "off by one", "reversed", "packed"])
@pytest.mark.parametrize("width", [40, 600, 1100, 4096, 5000])
def test_layouts_give_the_same_bits_as_others(how, width):
    """Results hang on the values and on whether they lie in whole vectors, not on where they lie; both are within the bounds above"""
    for kind in KIND:
        x, g, w = made((3, 4), width, kind, 1, 1.0), made((3, 4), width, kind, 2), factors(width, kind, 3, 1.0)
        b = factors(width, "float", 4, 0.0)

        def laid(t):
            t = t.cuda()
            return t.flip(0).flip(0) if how == "reversed" else spread(t, how)

        def turned(t):       # a view with a negative stride along the first dimension
            v = view(t)
            return ocn.Tensor(v.base + (t.shape[0] - 1) * v.strides[0], v.dtype, v.sizes, (-v.strides[0],) + v.strides[1:], 0, v.device, t)

        see = turned if how == "reversed" else view
        a, ga, out, gin = laid(x), laid(g), laid(torch.zeros_like(x)), laid(torch.zeros_like(x))
        gw, gb = torch.zeros(width, device="cuda"), torch.zeros(width, device="cuda")
        weight = torch.zeros(width, 3, dtype=KIND[kind], device="cuda")[:, 1].copy_(w.cuda())
        ocn.layer_norm(see(a), view(weight), view(b.cuda()), see(out))
        ocn.layer_norm_grad(see(ga), see(a), view(weight), see(gin), view(gw), view(gb))
        xd, gd = x.double(), g.double()
        if how == "reversed":
            out, gin = out.flip(0).flip(0), gin
        u, r, shift, _ = parts(xd, 1e-5)
        off = bound_of_u(u, r, shift, xd, kind)
        want = u * w.double() + b.double()
        check(out, want, rounding(kind, want) + off * w.double().abs() + F32 * want.abs())
        h = gd * w.double()
        want = r * (h - h.mean(-1, keepdim=True) - u * (h * u).mean(-1, keepdim=True))
        mean_hu = (h * u).abs().mean(-1, keepdim=True)
        size = h.abs() + h.abs().mean(-1, keepdim=True) + u.abs() * mean_hu
        bound = r * (44 * F32 * size + off * mean_hu + u.abs() * (h.abs() * off).mean(-1, keepdim=True)) + want.abs() * (shift ** 2 + 30 * F32)
        check(gin, want, rounding(kind, want) + bound)
        kept = out.clone()
        ocn.layer_norm(see(a), view(weight), view(b.cuda()), see(a))                    # in place
        assert torch.equal(a, kept)
        a2, kept = laid(x), gin.clone()
        ocn.layer_norm_grad(see(ga), see(a2), view(weight), see(a2), view(gw), view(gb))  # in the place of x, and of the gradient
        assert torch.equal(a2, kept)
        a2 = laid(x)
        ocn.layer_norm_grad(see(ga), see(a2), view(weight), see(ga))
        assert torch.equal(ga, kept)


def test_gradient_against_differences():
    x, g, w, b = made((3,), 20, "float", 1), made((3,), 20, "float", 2), factors(20, "float", 3, 1.0), factors(20, "float", 4, 0.0)
    gin, gw, gb = torch.zeros_like(x).cuda(), torch.zeros(20).cuda(), torch.zeros(20).cuda()
    ocn.layer_norm_grad(view(g.cuda()), view(x.cuda()), view(w.cuda()), view(gin), view(gw), view(gb))

    def f(x, w, b):
        u, _, _, _ = parts(x, 1e-5)
        return ((u * w + b) * g.double()).sum().item()

    at = [x.double(), w.double(), b.double()]
    step = 1e-6
    for n, got in enumerate((gin, gw, gb)):
        for i in range(at[n].numel()):
            e = torch.zeros(at[n].numel(), dtype=torch.float64)
            e[i] = step
            up, down = ([t + s * e.view(t.shape) if m == n else t for m, t in enumerate(at)] for s in (1, -1))
            # (differences of sums of some 60 are off by 1e-14 / step, the formula by step^2; single precision by 1e-6 of results up to 10)
            assert abs((f(*up) - f(*down)) / (2 * step) - got.flatten()[i].item()) < 1e-5


def test_rows_far_from_zero():
    """x = 1000 + small: the variance is that of the small part"""
    small = made((4,), 777, "float", 3)
    x = 1000 + small
    out = torch.zeros_like(x).cuda()
    ocn.layer_norm(view(x.cuda()), None, None, view(out))
    u, r, _, _ = parts(x.double(), 1e-5)
    # a deviation from the first mean (itself off by up to 40 half steps of 1000) is exact or rounded once, the mean of the deviations gives the rest
    check(out, u, rounding("float", u) + 60 * F32 * (u.abs() + 0.01) + 44 * F32 * 40 * F32 * 1000 * r)


def test_extreme_rows():
    """Constant rows, infinities and NaN stay in their rows"""
    for width in (64, 1500, 6000, 10000):
        x = made((6,), width, "float")
        x[0] = 3.0
        x[2, 5] = float("nan")
        x[4, 9] = float("inf")
        out, gin = torch.zeros_like(x).cuda(), torch.zeros_like(x).cuda()
        ocn.layer_norm(view(x.cuda()), None, None, view(out))
        ocn.layer_norm_grad(view(made((6,), width, "float", 1).cuda()), view(x.cuda()), None, view(gin))
        for t in (out.cpu(), gin.cpu()):
            assert t[2].isnan().all() and t[4].isnan().all() and t[[0, 1, 3, 5]].isfinite().all()
        assert (out[0].cpu().abs() <= 2e-4).all()       # (3 less its own mean, which is off by 40 half steps of 3 at most, over sqrt(eps))


def test_again_and_in_a_graph():
    """The same bits every time, in a graph too, between other calls"""
    x, g, w, b = made((3000,), 1280, "bfloat16", 1).cuda(), made((3000,), 1280, "bfloat16", 2).cuda(), factors(1280, "bfloat16", 3, 1.0).cuda(), factors(1280, "float", 4, 0.0).cuda()
    outs = [torch.zeros_like(x), torch.zeros_like(x), torch.zeros(1280, device="cuda"), torch.zeros(1280, device="cuda")]
    space = torch.empty(ocn.layer_norm_grad_workspace_bytes(view(x)), dtype=torch.uint8, device="cuda")

    def call():
        ocn.layer_norm(view(x), view(w), view(b), view(outs[0]))
        ocn.layer_norm_grad(view(g), view(x), view(w), view(outs[1]), view(outs[2]), view(outs[3]), workspace=space)

    call()
    first = [t.clone() for t in outs]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        for t in outs:
            t.fill_(7)
        space.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, outs))


def test_many_rows_over_a_capped_grid():
    from paper_1810_08723_amd import binding
    for width in (40, 4096):
        x = made((401,), width, "half").cuda()
        want, got = torch.zeros_like(x), torch.zeros_like(x)
        ocn.layer_norm(view(x), None, None, view(want))
        binding.set_max_launch_blocks(3)
        try:
            ocn.layer_norm(view(x), None, None, view(got))
            torch.cuda.synchronize()
        finally:
            binding.set_max_launch_blocks(0)
        assert torch.equal(want, got)


def test_another_stream_and_a_workspace_of_its_own():
    x, g = made((500,), 300, "half", 1).cuda(), made((500,), 300, "half", 2).cuda()
    w = factors(300, "half", 3, 1.0).cuda()
    want, wb = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda")
    gin = torch.zeros_like(x)
    ocn.layer_norm_grad(view(g), view(x), view(w), view(gin), view(want), view(wb))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, gb, gin2 = torch.zeros(300, device="cuda"), torch.zeros(300, device="cuda"), torch.zeros_like(x)
    torch.cuda.synchronize()
    ocn.layer_norm_grad(view(g), view(x), view(w), view(gin2), view(got), view(gb), stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(gb, wb) and torch.equal(gin, gin2)


def test_no_rows():
    """Gradients of factors are zeros where there are no rows"""
    x = torch.zeros(0, 100, device="cuda")
    gw, gb = torch.full((100,), 7.0, device="cuda"), torch.full((100,), 7.0, dtype=torch.bfloat16, device="cuda")
    ocn.layer_norm_grad(view(x), view(x), view(torch.ones(100, device="cuda")), view(torch.zeros(0, 100, device="cuda")), view(gw), view(gb))
    assert (gw == 0).all() and (gb == 0).all()
