"""Attention over whole sequences and its gradient where blocks, scores or values are out of the ordinary, against the forms and bounds of attention_ref."""
import math

import pytest
import torch

import paper_1810_08723_amd as ocn
from attention_ref import seen
from heads_ref import F32, KIND, half_step, view
from test_gpu_attention import both, check, close, made, reference, starts_of

pytestmark = pytest.mark.gpu

# blocks of keys that no query sees, beside ordinary ones: sequences without queries, windows that begin behind the first keys
UNSEEN = [([0, 40, 0, 7, 200], [300, 40, 500, 260, 30], 4, 2, 128, True, 0), ([0, 40, 0, 7, 200], [300, 40, 500, 260, 30], 4, 2, 128, True, 50),
          ([3, 0, 5], [2000, 700, 5], 2, 1, 128, True, 64), ([0, 30], [300, 70], 4, 4, 112, False, 0), ([0, 9], [600, 400], 2, 1, 192, True, 20), ([0, 9], [600, 400], 2, 1, 256, True, 20)]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", UNSEEN, ids=str)
def test_keys_that_no_query_sees(shape, kind):
    data = made(shape, kind, 30)
    got = both(shape, kind, data)
    check(shape, kind, data, got)
    if shape[0][0] == 0:
        assert all((got[n][:shape[1][0]] == 0).all() for n in ("gk", "gv"))


@pytest.mark.parametrize("scale", [1e-44, 1e-46, -1e-46, 1e-300, -5e-324])
def test_scales_below_single_precision(scale):
    """All keys that a query sees weigh the same; keys that it does not see weigh nothing.  (The scale itself is off by half of single precision's least number where gradients are multiplied by it.)"""
    shape = ([70, 5, 300], [70, 40, 300], 4, 2, 64, True, 0)
    for kind in KIND:
        data = made(shape, kind, 31)
        got = both(shape, kind, data, scale)
        want = reference(shape, kind, data, scale, got["out"].cpu())
        for n in got:
            value, bound = want[n]
            if n in ("gq", "gk"):
                bound = bound + 2.0 ** -150 * (1 + (value / scale).abs())
            close(n, got[n], (value, bound), None if n == "log_sum" else kind)


def gradient_of(p, q, k, v, w, out, scale, kind):
    """Gradients in 64 bits for weights p [heads, queries, keys] of one sequence, and how far the framework's may be from them where each weight that is not zero is right
    to 32 half steps of single precision: D is taken from out as it was rounded, at worst"""
    u, t = F32, (0.0 if kind == "float" else half_step(kind))
    tiny = 2.0 ** -36 if kind == "half" else 0.0
    group = q.shape[1] // k.shape[1]
    q, w, out = (x.double().transpose(0, 1) for x in (q, w, out))
    k, v = (x.double().transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
    d, rows = q.shape[2], q.shape[0] // (k.shape[0] // group) * q.shape[1]
    dp, size = w @ v.transpose(1, 2), w.abs() @ v.abs().transpose(1, 2)
    along = (p * dp).sum(2, keepdim=True)
    c = p * (dp - along)
    along_off = 2 * (t + F32) * (w.abs() * out.abs()).sum(2, keepdim=True) + (p.shape[2] + d + 64) * u * (p * size).sum(2, keepdim=True)
    c_off = 1.01 * (p * ((d + 2) * u * size + along_off) + (t + 64 * u) * c.abs())
    c_off = c_off + tiny * c_off.amax() + tiny * c.abs().amax()
    gq, gk, gv = scale * (c @ k), scale * (c.transpose(1, 2) @ q), p.transpose(1, 2) @ w
    gq_off = abs(scale) * (c_off @ k.abs() + (p.shape[2] + 4) * u * (c.abs() @ k.abs()))
    gk_off = abs(scale) * (c_off.transpose(1, 2) @ q.abs() + (rows + 4) * u * (c.abs().transpose(1, 2) @ q.abs()))
    gv_off = (p * (t + 32 * u) + tiny).transpose(1, 2) @ w.abs() + (rows + 4) * u * (p.transpose(1, 2) @ w.abs())
    of_head = lambda x: x.view(-1, group, *x.shape[1:]).sum(1).transpose(0, 1)
    return {"gq": (gq.transpose(0, 1), gq_off.transpose(0, 1)), "gk": (of_head(gk), of_head(gk_off)), "gv": (of_head(gv), of_head(gv_off))}


def largest_alone(s):
    """Weights of scores of which the largest ones are the same, and others so far below that they weigh nothing"""
    best = s == s.amax(2, keepdim=True)
    rest = torch.where(best, -math.inf, s).amax(2)
    assert ((s.amax(2) - rest) > 110).all()
    return best.double() / best.sum(2, keepdim=True)


@pytest.mark.parametrize("kind,size,scale", [("half", 200.0, 10.0), ("half", 60000.0, 0.1), ("bfloat16", 1e9, 1.0), ("bfloat16", 1e15, -1.0), ("float", 3000.0, 1.0), ("float", 1e12, -1.0),
                                             ("bfloat16", 1e-20, 1e32), ("float", 1e30, 1e20), ("bfloat16", 1e30, -1e20)])
@pytest.mark.parametrize("queries,keys", [(1, 200), (50, 200), (300, 900), (700, 90)])
@pytest.mark.parametrize("sign", [1, -1])
def test_gradients_of_scores_of_any_size(kind, size, scale, queries, keys, sign):
    """One channel of queries that is not zero, so that scores are exact, and keys that differ by a tenth there: the largest have all the weight, however large scores are, or how far below zero"""
    d, g = 64, torch.Generator().manual_seed(32)
    q, k, v, w = torch.zeros(queries, 2, d), torch.randn(keys, 1, d, generator=g), torch.randn(keys, 1, d, generator=g), torch.randn(queries, 2, d, generator=g)
    q[..., 0] = size
    k[:, 0, 0] = torch.linspace(0.125, 1.625, 16)[torch.randint(0, 16, (keys,), generator=g)] * sign
    data = tuple(t.to(KIND[kind]) for t in (q, k, v, w))
    got = both(([queries], [keys], 2, 1, d, False, 0), kind, data, scale)
    q, k, v, w = data
    p = largest_alone((q.double()[..., 0].t()[..., None] * k.double()[:, 0, 0]) * scale)
    want = gradient_of(p, q, k, v, w, got["out"].cpu(), scale, kind)
    out = (p @ v.double()[:, 0]).transpose(0, 1)
    close("out", got["out"], (out, (half_step(kind) + (keys + 64) * F32) * (p @ v.double()[:, 0].abs()).transpose(0, 1)), kind)
    most = torch.finfo(KIND[kind]).max / 2
    for n, (value, off) in want.items():
        fits = (value.abs() + off < most) & (value.abs() + off < 1e38)
        assert n == "gk" or fits.all()
        close(n, torch.where(fits.cuda(), got[n], 0), tuple(torch.where(fits, x, 0.0) for x in (value, off)), kind)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("n,heads,kv,d,window", [(40, 2, 2, 64, 0), (300, 4, 2, 128, 0), (700, 4, 1, 128, 0), (500, 2, 1, 80, 150), (90, 3, 1, 192, 0), (350, 2, 2, 256, 0), (400, 2, 1, 100, 0)])
def test_gradients_of_far_scores(kind, n, heads, kv, d, window):
    """Scores of all channels up to 1e11: a row's largest key has all of its weight, which is one in both passes where they make the same score of it"""
    scale, shape = 1e9, ([n], None, heads, kv, d, True, window)
    q, k, v, w = data = made(shape, kind, 33)
    s = (q.double().transpose(0, 1) @ k.double().transpose(0, 1).repeat_interleave(heads // kv, 0).transpose(1, 2) * scale).masked_fill(~seen(n, n, True, window), -math.inf)
    size = q.double().abs().transpose(0, 1) @ k.double().abs().transpose(0, 1).repeat_interleave(heads // kv, 0).transpose(1, 2) * scale
    gaps = s.topk(2, 2).values.diff(dim=2).neg()
    clear = (gaps[..., 0] > 4 * (d + 2) * F32 * size.amax(2)) | (torch.arange(n) == 0)
    data = (q, k, v, w) = (q, k, v, w * clear.t()[..., None].to(w.dtype))          # (rows whose largest two are too near to each other for single precision have no part in it)
    assert clear.double().mean() > 0.9
    got = both(shape, kind, data, scale)
    want = gradient_of(largest_alone(torch.where(clear[..., None], s, torch.where(torch.arange(n) == 0, 0.0, -math.inf))), q, k, v, w, got["out"].cpu(), scale, kind)
    for name, (value, off) in want.items():
        fits = value.abs() + off < torch.finfo(KIND[kind]).max / 2
        if name == "gq":
            fits = fits & clear.t()[..., None]
        close(name, torch.where(fits.cuda(), got[name], 0), tuple(torch.where(fits, x, 0.0) for x in (value, off)), kind)
        assert name != "gv" or fits.all()


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d", [64, 128, 192])
def test_a_single_key(kind, d):
    """A window of one: the gradient of a value is that of its query's result, at any scale.  (In single precision the exponent of a weight is off by four half steps of 128 at most.)"""
    shape = ([300, 7], None, 2, 2, d, True, 1)
    data = made(shape, kind, 34)
    for scale in (0.1, 1e3, -1e6, 1e9, 1e20):
        got = both(shape, kind, data, scale)
        assert torch.equal(got["out"].cpu(), data[2])
        assert ((got["gv"].cpu().double() - data[3].double()).abs() <= (360 * F32 if kind == "float" else 0.0) * data[3].double().abs()).all(), scale


@pytest.mark.parametrize("kind", list(KIND))
def test_far_scores_of_sequences_as_a_dimension(kind):
    """[batch, tokens, heads, channels], heads first in memory: a single key again; and the same bits in several launches, on another stream and from a workspace of anything"""
    from paper_1810_08723_amd import binding
    batch, n, heads, d = 3, 150, 4, 128
    q, k, v, w = (t.cuda().view(batch, n, heads, d).transpose(1, 2).contiguous().transpose(1, 2) for t in made(([batch * n], None, heads, heads, d, True, 0), kind, 41))

    def run(window, scale, stream=None):
        r = {"out": torch.zeros_like(q), "log_sum": torch.zeros(batch, n, heads, device="cuda"), "gq": torch.zeros_like(q), "gk": torch.zeros_like(k), "gv": torch.zeros_like(v)}
        vr = {name: view(t) for name, t in r.items()}
        space = torch.full((ocn.attention_grad_workspace_bytes(view(q), view(k)),), 255, dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        ocn.attention(view(q), view(k), view(v), vr["out"], scale, window=window, log_sum=vr["log_sum"], stream=stream)
        ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], scale, window=window, workspace=space, stream=stream)
        torch.cuda.synchronize()
        return r

    got = run(1, 1e9)
    assert torch.equal(got["out"], v) and torch.equal(got["gv"], w)
    first = run(0, 1e9)
    assert all(t.isfinite().all() for name, t in first.items() if kind != "half" or name in ("out", "log_sum", "gv"))
    binding.set_max_launch_blocks(3)
    try:
        again = run(0, 1e9)
    finally:
        binding.set_max_launch_blocks(0)
    other = run(0, 1e9, torch.cuda.Stream().cuda_stream)
    assert all(torch.equal(first[name].nan_to_num(), x[name].nan_to_num()) for name in first for x in (again, other))


@pytest.mark.parametrize("kind", list(KIND))
def test_one_row_of_far_scores(kind):
    for shape in (([90], None, 2, 1, 64, True, 0), ([700], None, 4, 2, 128, True, 0)):
        q, k, v, w = made(shape, kind, 35)
        q[60, 1] *= 300
        check(shape, kind, (q, k, v, w), both(shape, kind, (q, k, v, w)))


def reached(shape, rows=None, keys=None):
    """[queries, keys] of the last sequence: whether a query that is among the rows, or sees one of the keys, sees the key"""
    n = shape[0][-1]
    see = seen(n, n, True, shape[6])
    hit = torch.zeros(n, dtype=torch.bool)
    if rows is not None:
        hit[rows] = True
    if keys is not None:
        hit |= see[:, keys].any(1)
    return hit, (see & hit[:, None]).any(0)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("d", [64, 80, 128, 256])
@pytest.mark.parametrize("n", [100, 900])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_what_is_no_number_in_one_operand(kind, d, n, bad):
    """A NaN or an infinity in one operand alone of one sequence: gradients are NaN wherever the definition's are, and those of other sequences are as they were"""
    shape = ([70, n], None, 4, 2, d, True, 0)
    data = made(shape, kind, 36)
    plain = both(shape, kind, data)
    row, first = n // 2, 70
    for which in range(4):
        tensors = [t.clone() for t in data]
        tensors[which][first + row, 1, 3] = bad
        got = {name: t.cpu() for name, t in both(shape, kind, tensors).items()}
        assert all(torch.equal(got[name][:first], plain[name].cpu()[:first]) for name in got)
        # head 1 of the queries reads head 0 of the keys; head 1 of the keys is read by the heads 2 and 3
        of_query = which in (0, 3)
        hit, held = reached(shape, rows=[row]) if of_query else reached(shape, keys=[row])
        heads, kv = ([1], 0) if of_query else ([2, 3], 1)
        gk, gv = got["gk"][first:, kv][held], got["gv"][first:, kv][held]
        for h in heads:
            gq = got["gq"][first:, h][hit]
            # (an infinity of a key makes scores of minus infinity too, weights of zero, and NaNs of those times itself)
            assert (gq if which != 1 or bad != bad else gq[:, 3]).isnan().all(), (which, "gq")
        if bad != bad:
            assert gk.isnan().all() and (which not in (0, 1) or gv.isnan().all()) and (which != 3 or gv[:, 3].isnan().all()), which
        elif which >= 2:
            assert not gk.isfinite().any() and (which != 3 or not gv[:, 3].isfinite().any()), which


@pytest.mark.parametrize("kind", ["bfloat16", "float"])
@pytest.mark.parametrize("n", [100, 900])
def test_scores_that_are_no_numbers(kind, n):
    """Finite queries and keys whose products pass single precision: results that are NaN have gradients that are"""
    shape = ([70, n], None, 2, 1, 64, True, 0)
    q, k, v, w = made(shape, kind, 37)
    q[70 + n // 2, 0] = 1e30
    k[70 + n // 4, 0] = 1e30
    got = {name: t.cpu() for name, t in both(shape, kind, (q, k, v, w)).items()}
    odd = got["out"].isnan().any(2)
    assert odd[70 + n // 2, 0] and odd.sum() == 1
    assert got["gq"][70 + n // 2, 0].isnan().all()
    for name in ("gk", "gv"):
        assert got[name][70:70 + n // 2 + 1].isnan().all()
        assert got[name][:70].isfinite().all()


def with_odd_values(v, share, seed):
    """v with NaNs and infinities, in whole keys of the first heads and here and there"""
    g = torch.Generator().manual_seed(seed)
    v = v.clone()
    what = torch.tensor([math.nan, math.inf, -math.inf]).to(v.dtype)[torch.randint(0, 3, v.shape, generator=g)]
    where = torch.rand(v.shape, generator=g) < share
    where[:, 0] &= torch.rand(len(v), 1, generator=g) < 0.3
    return torch.where(where, what, v)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("share", [0.0005, 0.05, 1.0])
@pytest.mark.parametrize("shape", [([130, 40], None, 4, 2, 64, True, 0), ([700], None, 2, 2, 128, True, 200), ([90], [300], 4, 2, 80, False, 0), ([1, 3, 1], [70, 300, 1500], 8, 2, 128, True, 33),
                                   ([2], [3000], 4, 1, 100, True, 0), ([150], None, 2, 1, 192, True, 0), ([77], None, 3, 3, 256, True, 30), ([200], [2500], 2, 1, 64, True, 0)], ids=str)
def test_values_that_are_no_numbers(shape, share, kind):
    """Results have what the values that a query sees have, channel by channel: a NaN or infinities of both signs make a NaN, an infinity itself, and without them they are those of numbers alone"""
    q, k, v, w = made(shape, kind, 38)
    v = with_odd_values(v, share, 39)
    got = both(shape, kind, (q, k, v, w), grad=False)
    number = v.float().isfinite()
    finite = reference(shape, kind, (q, k, torch.where(number, v, torch.zeros_like(v)), w), grad=False)
    nq, nk, heads, kv, d, causal, window = shape
    want, bound = (x.clone() for x in finite["out"])
    at_q = at_k = 0
    for n, m in zip(nq, nq if nk is None else nk):
        see = seen(n, m, causal, window).float()
        for h in range(heads):
            x = v[at_k:at_k + m, h * kv // heads].float()
            nan, up, down = (see @ y.float() > 0 for y in (x.isnan(), x == math.inf, x == -math.inf))
            rows = want[at_q:at_q + n, h]
            rows[up], rows[down], rows[nan | up & down] = math.inf, -math.inf, math.nan
        at_q, at_k = at_q + n, at_k + m
    out = got["out"].double().cpu()
    assert torch.equal(out.isnan(), want.isnan())
    close("out", torch.where(want.isnan(), 0.0, out), (torch.where(want.isnan(), 0.0, want), bound), kind)
    close("log_sum", got["log_sum"], finite["log_sum"], None)


@pytest.mark.parametrize("kind", list(KIND))
def test_values_that_are_all_nan_take_no_longer(kind):
    """As after a step that went astray: not key by key (1200 times as long), but within a few times of numbers"""
    shape = ([2000], None, 4, 1, 128, True, 0)
    q, k, v, _ = (t.cuda() for t in made(shape, kind, 40))
    out, s = torch.zeros_like(q), starts_of([2000]).cuda()
    times = []
    for values in (v, torch.full_like(v, math.nan)):
        best = math.inf
        for _ in range(5):
            begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            begin.record()
            for _ in range(4):
                ocn.attention(view(q), view(k), view(values), view(out), 0.1, view(s), view(s))
            end.record()
            torch.cuda.synchronize()
            best = min(best, begin.elapsed_time(end))
        times.append(best)
    assert out.isnan().all()
    assert times[1] <= 10 * times[0], times
