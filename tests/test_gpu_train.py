"""The layer of examples/train.py: every operator in it against its 64-bit form, its gradients against those of the whole layer in 64 bits, and a captured step."""
import math
import os
import sys

import pytest
import torch

from attention_ref import attended, spans
from heads_ref import F32, KIND, rounding
from test_gpu_axes import turned

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
pytestmark = pytest.mark.gpu
SHAPES = [(2, 3, 4), (1, 1, 1), (3, 5, 7), (1, 6, 6)]


def made(kind, causal=True, window=0, width=96, heads=4, kv=2, channels=32, pairs=(6, 5, 5)):
    from train import Layer, grids
    torch.manual_seed(1)
    layer = Layer(width, heads, kv, channels, pairs, KIND[kind], causal, window)
    with torch.no_grad():
        for p in (layer.weight, layer.bias, layer.q_weight, layer.k_weight):
            p.add_(0.2 * torch.randn(p.shape, device="cuda").to(p.dtype))
    positions, starts = grids(SHAPES)
    x = torch.randn(positions.shape[1], width, device="cuda").to(KIND[kind]).requires_grad_()
    return layer, x, positions, starts


def plain(layer, x, p, positions, starts):
    """The layer in 64 bits on the CPU, by torch's own operations; p: its parameters"""
    heads, kv, channels = layer.heads
    over = lambda t, w: t / (t.square().mean(-1, keepdim=True) + layer.eps).sqrt() * w  # noqa: E731
    mean = x.mean(-1, keepdim=True)
    h = over(x - mean, p["weight"]) + p["bias"]
    q, k, v = (h @ p["qkv"]).view(-1, heads + 2 * kv, channels).split([heads, kv, kv], dim=1)
    angle = (positions.double()[..., None] * layer.frequencies.cpu()[:, None]).sum(0)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    n = layer.rotary_dim // 2
    turn = lambda t: torch.cat([t[..., :n] * c - t[..., n:2 * n] * s, t[..., n:2 * n] * c + t[..., :n] * s, t[..., 2 * n:]], -1)  # noqa: E731
    q, k = turn(over(q, p["q_weight"])), turn(over(k, p["k_weight"]))
    outs = []
    for a, b in zip(starts[:-1].tolist(), starts[1:].tolist()):
        score = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(heads // kv, 1)) / math.sqrt(channels)
        i, j = torch.arange(b - a)[:, None], torch.arange(b - a)[None]
        if layer.causal:
            score = score.masked_fill(j > i, -math.inf)
            if layer.window:
                score = score.masked_fill(j <= i - layer.window, -math.inf)
        outs.append(torch.einsum("hij,jhd->ihd", score.softmax(-1), v[a:b].repeat_interleave(heads // kv, 1)))
    return x + torch.cat(outs).flatten(1) @ p["out"]


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 10)])
def test_gradients_of_the_layer(causal, window):
    """In single precision.  The longest sum has 192 terms (tokens of a weight's gradient: 166) and there are nine operators each way, so that an error of 9 * 2 * 192 u = 2^-12 in the
    norm is what sums in the worst order come to where no operator magnifies its input's; the norms of heads and rows divide by numbers near one, and softmax has scores below 11 (|q| |k| / sqrt d), whose
    errors it doubles.  2^-10 of a gradient's norm is four times that, and a term that is left out or a wrong factor is more."""
    layer, x, positions, starts = made("float", causal, window)
    w = torch.randn(x.shape, device="cuda")
    (layer(x, positions, starts) * w).sum().backward()
    p = {n: t.detach().double().cpu().requires_grad_() for n, t in layer.named_parameters()}
    xd = x.detach().double().cpu().requires_grad_()
    loss = (plain(layer, xd, p, positions.cpu(), starts.cpu()) * w.double().cpu()).sum()
    loss.backward()
    for name, got, want in [("x", x.grad, xd.grad)] + [(n, t.grad, p[n].grad) for n, t in layer.named_parameters()]:
        assert (got.double().cpu() - want).norm() <= 2.0 ** -10 * want.norm(), name
    # ... and of the 64-bit form along a direction, by differences
    g = torch.Generator().manual_seed(3)
    at = {"x": xd.detach(), **{n: t.detach() for n, t in p.items()}}
    way = {n: torch.randn(t.shape, generator=g, dtype=torch.float64) for n, t in at.items()}

    def f(step):
        m = {n: t + step * way[n] for n, t in at.items()}
        return (plain(layer, m.pop("x"), m, positions.cpu(), starts.cpu()) * w.double().cpu()).sum().item()

    grads = {"x": x.grad, **{n: t.grad for n, t in layer.named_parameters()}}
    along = sum((way[n] * grads[n].double().cpu()).sum().item() for n in way)
    size = sum((way[n].norm() * grads[n].double().cpu().norm()).item() for n in way)
    assert abs((f(1e-6) - f(-1e-6)) / 2e-6 - along) <= 2.0 ** -10 * size


@pytest.mark.parametrize("kind", list(KIND))
def test_operators_one_after_the_other(kind):
    """Each operator's results against the 64-bit form of what it was given, which the operator before it left"""
    from train import Attention, LayerNorm, NormRotary
    import paper_1810_08723_amd as ocn
    from train import view
    layer, x, positions, starts = made(kind)
    heads, kv, channels = layer.heads
    with torch.no_grad():
        h = LayerNorm.apply(x, layer.weight, layer.bias, layer.eps)
        xd = x.double().cpu()
        d = xd - xd.mean(-1, keepdim=True)
        u = d / (d.square().mean(-1, keepdim=True) + layer.eps).sqrt()
        want = u * layer.weight.double().cpu() + layer.bias.double().cpu()
        # the mean is off by 2 u of the largest, the sum of squares by (n + 2) u, and three roundings: all of it below (n + 16) u of sizes up to |u| and |x| / deviation
        size = (u.abs() + 1 + xd.abs().amax(-1, keepdim=True) / d.square().mean(-1, keepdim=True).sqrt()) * layer.weight.double().cpu().abs() + layer.bias.double().cpu().abs()
        assert ((h.double().cpu() - want).abs() <= rounding(kind, want) + (x.shape[1] + 16) * F32 * size).all()
        qkv = (h @ layer.qkv).view(-1, heads + 2 * kv, channels)
        q, k, v = qkv.split([heads, kv, kv], dim=1)
        rotation = ocn.Rotation(view(positions), view(layer.frequencies), layer.rotary_dim, "half", layer.magnitude)
        turned_heads = []
        for t, w in ((q, layer.q_weight), (k, layer.k_weight)):
            got = NormRotary.apply(t, w, rotation, layer.eps)
            td = t.double().cpu()
            normed = td / (td.square().mean(-1, keepdim=True) + layer.eps).sqrt() * w.double().cpu()
            want, size = turned(normed, positions.cpu(), layer.frequencies.cpu(), False)
            assert ((got.double().cpu() - want).abs() <= rounding(kind, want) + (channels + 16) * F32 * size).all()
            turned_heads.append(got)
        q, k = turned_heads
    q, k, v = (t.detach().clone().requires_grad_() for t in (q, k, v))
    scale = 1 / math.sqrt(channels)
    out = Attention.apply(q, k, v, starts, scale, True, 0)
    gout = torch.randn(out.shape, device="cuda").to(out.dtype)
    out.backward(gout)
    sp = spans(starts.cpu(), len(q))
    want = attended(q.detach().cpu(), k.detach().cpu(), v.detach().cpu(), sp, sp, scale, True, 0, kind, gout.cpu(), out.detach().cpu())
    for name, got in (("out", out), ("gq", q.grad), ("gk", k.grad), ("gv", v.grad)):
        value, bound = want[name]
        assert ((got.detach().double().cpu() - value).abs() <= bound + rounding(kind, value)).all(), name


def test_a_captured_step_and_an_eager_one():
    """Forward and backward in a graph, replayed with eager steps of another layer between: the bits of an eager step, with leaves of its own"""
    layer, x, positions, starts = made("bfloat16")
    w = torch.randn(x.shape, device="cuda").to(x.dtype)

    def step(leaves_of, at):
        leaves = [at] + list(leaves_of.parameters())
        return [leaves_of(at, positions, starts)] + list(torch.autograd.grad(leaves_of(at, positions, starts), leaves, w))

    other, y, _, _ = made("bfloat16")
    eager = [t.detach().clone() for t in step(other, y)]
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        for _ in range(2):
            step(layer, x)
    torch.cuda.current_stream().wait_stream(warm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(layer, x)
    for _ in range(3):
        for t in got:
            t.detach().fill_(7)
        graph.replay()
        again = step(other, y)
        torch.cuda.synchronize()
        assert all(torch.equal(a.detach(), b) for a, b in zip(got, eager))
        assert all(torch.equal(a.detach(), b) for a, b in zip(again, eager))


def test_sequences_are_apart():
    """A sequence's results and gradients are those that it has by itself, bit for bit, whatever the others hold: NaNs among it"""
    from train import Attention
    torch.manual_seed(2)
    for channels, dtype in ((64, torch.float16), (128, torch.bfloat16), (80, torch.float16), (192, torch.bfloat16)):
        lengths = [70, 33, 1, 150]
        starts = torch.tensor([0] + lengths).cumsum(0).to("cuda", torch.int32)
        q, k, v, w = (torch.randn(sum(lengths) + 5, h, channels, device="cuda").to(dtype) for h in (4, 2, 2, 4))
        results = []
        for odd in (False, True):
            ts = [t.clone() for t in (q, k, v)]
            for t in ts:
                if odd:
                    t[starts[1]:starts[2]] = math.nan
                    t[starts[3] + 149 + 1:] = math.inf
                t.requires_grad_()
            gout = w.clone()
            out = Attention.apply(*ts, starts, 0.1, True, 0)
            if odd:
                gout[starts[1]:starts[2]] = math.nan
                gout[starts[4]:] = math.nan
            # (rows of no sequence: whatever the buffers held)
            results.append([t[:starts[4]] for t in (out.detach(), *torch.autograd.grad(out, ts, gout))])
        own = torch.ones(sum(lengths), dtype=torch.bool, device="cuda")
        own[starts[1]:starts[2]] = False
        for a, b in zip(*results):
            assert a[own].isfinite().all() and torch.equal(a[own], b[own])
            assert b[~own].isnan().all()


def test_the_example_runs():
    import train
    argv, sys.argv = sys.argv, ["train.py", "--sequences", "2", "--longest", "512", "--steps", "2"]
    try:
        train.main()
    finally:
        sys.argv = argv
