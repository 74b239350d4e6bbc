"""Attention over whole sequences and its gradient against the 64-bit forms and bounds of attention_ref."""
import math

import pytest
import torch

import paper_1810_08723_amd as ocn
from attention_ref import attended, spans
from heads_ref import KIND, rounding, view
from test_gpu_heads import spread

pytestmark = pytest.mark.gpu

# lengths of queries, of keys (None: the same), heads, kv heads, channels, causal, window
SHAPES = [([1], None, 1, 1, 64, True, 0), ([5, 1, 17], None, 4, 2, 64, True, 0), ([33, 0, 64, 2], None, 8, 2, 128, True, 0), ([40], None, 3, 1, 80, False, 0),
          ([130, 3], None, 7, 1, 32, True, 0), ([100, 31], None, 2, 2, 17, True, 9), ([65], None, 4, 4, 96, False, 0), ([70, 29], None, 2, 1, 192, True, 0),
          ([66], None, 2, 1, 256, True, 40), ([31, 20], None, 5, 5, 250, False, 0), ([300, 7], None, 8, 2, 128, True, 64), ([257], None, 6, 2, 64, True, 0),
          ([1, 1, 1], [70, 0, 513], 8, 2, 128, True, 0), ([1] * 5, [1, 2, 33, 64, 300], 4, 4, 64, True, 0), ([3, 2], [200, 40], 16, 2, 128, True, 50),
          ([4, 9], [2, 3], 4, 2, 64, True, 0), ([50, 20], [20, 77], 4, 2, 128, False, 0), ([37], [300], 6, 3, 100, True, 0), ([2], [1500], 40, 1, 64, True, 0),
          ([0, 3], [5, 0], 2, 1, 64, False, 0), ([20], None, 300, 2, 64, True, 0), ([1, 2], [90, 33], 1, 1, 160, True, 0), ([520], None, 1, 1, 128, True, 0)]


def starts_of(lengths, wide=False):
    return torch.tensor([sum(lengths[:i]) for i in range(len(lengths) + 1)], dtype=torch.int64 if wide else torch.int32)


def made(shape, kind, seed=0):
    nq, nk, heads, kv, d, _, _ = shape
    g = torch.Generator().manual_seed(seed)
    nk = nq if nk is None else nk
    q, k, v, w = (torch.randn(sum(n), h, d, generator=g).to(KIND[kind]) for n, h in ((nq, heads), (nk, kv), (nk, kv), (nq, heads)))
    return q, k, v, w


def close(name, got, want, kind):
    value, bound = want
    got = got.double().cpu()
    assert got.shape == value.shape
    there = ~value.isnan()
    same = (got == value) & there            # (infinities)
    bound = bound + (rounding(kind, value) if kind else 0.0)
    bad = there & ~same & ~((got - value).abs() <= bound)
    assert not bad.any(), (name, int(bad.sum()), ((got - value).abs() / bound)[bad].max().item(), bad.nonzero()[:3].tolist())


def both(shape, kind, data, scale=None, how="", wide=False, grad=True, fill=7.0):
    """The framework's results, on tensors laid out in some way: a dict"""
    nq, nk, heads, kv, d, causal, window = shape
    q, k, v, w = (spread(t.cuda(), how) for t in data)
    scale = 1 / math.sqrt(d) if scale is None else scale
    s = [starts_of(nq, wide).cuda(), starts_of(nq if nk is None else nk, wide).cuda()]
    r = {"out": spread(torch.full_like(q, fill), how), "log_sum": torch.full(q.shape[:2], fill, device="cuda")}
    arg = {"q_starts": view(s[0]), "k_starts": view(s[1]), "causal": causal, "window": window}
    ocn.attention(view(q), view(k), view(v), view(r["out"]), scale, log_sum=view(r["log_sum"]), **arg)
    if grad:
        r |= {n: spread(torch.full_like(t, fill), how) for n, t in (("gq", q), ("gk", k), ("gv", v))}
        ocn.attention_grad(view(w), view(q), view(k), view(v), view(r["out"]), view(r["log_sum"]), view(r["gq"]), view(r["gk"]), view(r["gv"]), scale, **arg)
    torch.cuda.synchronize()
    return r


def reference(shape, kind, data, scale=None, kept=None, grad=True):
    nq, nk, heads, kv, d, causal, window = shape
    q, k, v, w = data
    sq, sk = spans(starts_of(nq), len(q)), spans(starts_of(nq if nk is None else nk), len(k))
    return attended(q, k, v, sq, sk, 1 / math.sqrt(d) if scale is None else scale, causal, window, kind, w if grad else None, kept)


def check(shape, kind, data, got, scale=None):
    want = reference(shape, kind, data, scale, got["out"].cpu(), "gq" in got)
    for n in got:
        close(n, got[n], want[n], None if n == "log_sum" else kind)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_packed(shape, kind):
    data = made(shape, kind)
    check(shape, kind, data, both(shape, kind, data))


@pytest.mark.parametrize("how", ["packed", "channels", "heads first", "off by one"])
@pytest.mark.parametrize("shape", [SHAPES[2], SHAPES[3], SHAPES[5], SHAPES[12], SHAPES[17]], ids=str)
def test_layouts(shape, how):
    for kind in KIND:
        data = made(shape, kind, 1)
        check(shape, kind, data, both(shape, kind, data, how=how, wide=how == "packed"))


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 2.0])
def test_scales(scale):
    shape = ([70, 5], None, 4, 2, 64, True, 0)
    for kind in KIND:
        data = made(shape, kind, 2)
        check(shape, kind, data, both(shape, kind, data, scale), scale)


@pytest.mark.parametrize("kind", list(KIND))
def test_sequences_as_a_dimension(kind):
    """[batch, tokens, heads, channels], in the order of heads or of tokens, gives what packed sequences give"""
    for nq, nk, heads, kv, d, causal, window in ((37, 37, 4, 2, 64, True, 0), (1, 130, 8, 2, 128, True, 0), (20, 70, 3, 3, 40, False, 0), (150, 150, 2, 1, 128, True, 33)):
        shape = ([nq] * 3, [nk] * 3, heads, kv, d, causal, window)
        data = made(shape, kind, 3)
        packed = both(shape, kind, data)
        for heads_first in (False, True):
            def four(t, n):
                t = t.cuda().view(3, n, t.shape[1], d)
                return t.transpose(1, 2).contiguous().transpose(1, 2) if heads_first else t
            q, k, v, w = (four(t, n) for t, n in zip(data, (nq, nk, nk, nq)))
            r = {"out": torch.zeros_like(q), "log_sum": torch.zeros(3, heads, nq, device="cuda").transpose(1, 2), "gq": torch.zeros_like(q), "gk": torch.zeros_like(k), "gv": torch.zeros_like(v)}
            ocn.attention(view(q), view(k), view(v), view(r["out"]), 1 / math.sqrt(d), causal=causal, window=window, log_sum=view(r["log_sum"]))
            ocn.attention_grad(view(w), view(q), view(k), view(v), view(r["out"]), view(r["log_sum"]), view(r["gq"]), view(r["gk"]), view(r["gv"]), 1 / math.sqrt(d),
                               causal=causal, window=window)
            got = {n: t.reshape(packed[n].shape) for n, t in r.items()}
            check(shape, kind, data, got)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("queries", [None, 2])
def test_what_is_not_seen_does_not_reach_results(kind, queries):
    """Infinities and NaNs in keys and values, and in other sequences: rows that do not see them have the results that they have without"""
    for d in (64, 128, 256):
        lengths = [90, 40]
        shape = ([queries or n for n in lengths], lengths, 4, 2, d, True, 30 if d == 128 else 0)
        data = made(shape, kind, 4)
        want = both(shape, kind, data, grad=False)
        q, k, v, w = (t.clone() for t in data)
        for i, (t, bad) in enumerate(((k, float("nan")), (v, float("inf")), (v, float("nan")), (v, -float("inf")))):
            t[lengths[0] - 1 - 2 * i, i % 2, 3] = bad
        # keys past position 82 of the first sequence are odd: rows that see none of them
        got = both(shape, kind, (q, k, v, w), grad=False)
        ends = torch.cat([torch.arange(n - m + 1, n + 1) for n, m in zip(lengths, shape[0])])
        clean = torch.ones(len(q), dtype=torch.bool)
        clean[:shape[0][0]] = ends[:shape[0][0]] <= 83
        a, b = (r["out"][clean].double().cpu() for r in (want, got))
        ref = reference(shape, kind, data, grad=False)
        assert a.isfinite().all() and b.isfinite().all()
        close("out", got["out"].masked_fill(~clean.cuda()[:, None, None], 0.0), tuple(x.masked_fill(~clean[:, None, None], 0.0) for x in ref["out"]), kind)
        close("log_sum", got["log_sum"].masked_fill(~clean.cuda()[:, None], 0.0), tuple(x.masked_fill(~clean[:, None], 0.0) for x in ref["log_sum"]), None)
        last = got["out"][shape[0][0] - 1]       # sees all of them
        assert last.isnan().any()
        # one value of infinity alone: rows that see it have it, in its channel and no other
        v = data[2].clone()
        v[87, 0, 5] = float("inf")
        got = both(shape, kind, (data[0], data[1], v, w), grad=False)["out"].cpu()
        for i in range(shape[0][0]):
            sees = ends[i] > 87
            for h in range(4):
                row = got[i, h].clone()
                assert (row[5] == float("inf")) == bool(sees and h < 2)
                row[5] = 0
                assert row.isfinite().all()


def test_starts_outside_and_rows_of_no_sequence():
    """Starts are held to the tensor, and tokens before the first and behind the last sequence keep what the outputs hold"""
    for kind in KIND:
        shape = ([20, 30, 10], None, 4, 2, 64, True, 0)
        q, k, v, w = (t.cuda() for t in made(shape, kind, 5))
        for starts in ([7, 20, 20, 41], [-5, 10, 999, 10 ** 9]):
            s = torch.tensor(starts, dtype=torch.int64).cuda()
            r = {"out": torch.full_like(q, 7.0), "log_sum": torch.full(q.shape[:2], 7.0, device="cuda"), "gq": torch.full_like(q, 7.0), "gk": torch.full_like(k, 7.0), "gv": torch.full_like(v, 7.0)}
            ocn.attention(view(q), view(k), view(v), view(r["out"]), 0.2, view(s), view(s), log_sum=view(r["log_sum"]))
            ocn.attention_grad(view(w), view(q), view(k), view(v), view(r["out"]), view(r["log_sum"]), view(r["gq"]), view(r["gk"]), view(r["gv"]), 0.2, view(s), view(s))
            sp = spans(starts, 60)
            want = attended(q.cpu(), k.cpu(), v.cpu(), sp, sp, 0.2, True, 0, kind, w.cpu(), r["out"].cpu())
            for n in r:
                close(n, r[n], want[n], None if n == "log_sum" else kind)
                assert (r[n].cpu()[want[n][0].isnan()] == 7.0).all()


@pytest.mark.parametrize("kind,size,scale", [("half", 200.0, 1.0), ("half", 60000.0, 0.1), ("bfloat16", 1e9, 1.0), ("bfloat16", 1e15, -1.0), ("float", 1e12, 1.0), ("bfloat16", 1e-20, 1e32)])
@pytest.mark.parametrize("queries", [1, 50])
def test_scores_of_any_size(kind, size, scale, queries):
    """One channel that is not zero, so that scores are exact, and keys that differ by a tenth: the largest takes it all, however large scores are"""
    nk, d = 200, 64
    q, k = torch.zeros(queries, 2, d), torch.zeros(nk, 1, d)
    q[..., 0] = size
    k[:, 0, 0] = torch.linspace(-1, 1, 16)[torch.randint(0, 16, (nk,), generator=torch.Generator().manual_seed(1))]
    k[:3, 0, 0] = torch.tensor([1.0, -1.0, 1.0])
    q, k, v = (t.to(KIND[kind]) for t in (q, k, torch.randn(nk, 1, d, generator=torch.Generator().manual_seed(2))))
    s = [torch.tensor([0, n], dtype=torch.int32).cuda() for n in (queries, nk)]
    out, log = torch.zeros_like(q).cuda(), torch.zeros(queries, 2, device="cuda")
    ocn.attention(view(q.cuda()), view(k.cuda()), view(v.cuda()), view(out), scale, view(s[0]), view(s[1]), causal=False, log_sum=view(log))
    best = (k[:, 0, 0].double() * scale).max()
    mean = v[(k[:, 0, 0].double() * scale) == best][:, 0].double().mean(0)
    assert out.isfinite().all()
    assert ((out.double().cpu() - mean).abs() <= rounding(kind, mean) + 2.0 ** -15 * 4).all()
    want = best * q[0, 0, 0].double()
    assert ((log.double().cpu() - want).abs() <= 8 * 2.0 ** -24 * want.abs() + math.log(nk)).all()


@pytest.mark.parametrize("size", [1e-3, 1.0, 3e4])
def test_gradients_of_any_size_in_half(size):
    """Weights times differences of gout v pass a half's range, or lie below it: results are as exact as others"""
    shape = ([90, 33], None, 4, 2, 64, True, 0)
    q, k, v, w = made(shape, "half", 6)
    data = (q, k, (v.float() * 10).half(), (w.float().clamp(-2, 2) * size).half())
    got = both(shape, "half", data)
    want = reference(shape, "half", data, None, got["out"].cpu())
    for n in ("gq", "gk", "gv"):
        value, bound = want[n]
        fine = value.abs() < 65000
        close(n, torch.where(fine.cuda(), got[n], 0), tuple(torch.where(fine, x, 0.0) for x in (value, bound)), "half")


def test_gradient_against_differences():
    """The gradient of sum(out * w) by central differences of the 64-bit form"""
    shape = ([7, 4], [9, 4], 4, 2, 16, True, 0)
    data = made(shape, "float", 7)
    got = both(shape, "float", data)

    def f(q, k, v):
        r = reference(shape, "float", (q, k, v, data[3]), grad=False)["out"][0]
        return (r * data[3].double()).sum().item()

    at = [t.double() for t in data[:3]]
    step = 1e-5
    for n, name in enumerate(("gq", "gk", "gv")):
        flat = got[name].double().cpu().flatten()
        for i in range(0, len(flat), 11):
            e = torch.zeros(len(flat), dtype=torch.float64)
            e[i] = step
            up, down = ([t + s * e.view(t.shape) if m == n else t for m, t in enumerate(at)] for s in (1, -1))
            # (differences: step^2 and 1e-14 / step; single precision: some 1e-6 of values up to 10)
            assert abs((f(*up) - f(*down)) / (2 * step) - flat[i].item()) < 2e-5


def test_some_gradients():
    """Gradients that are not wanted are left out, the others have the same bits"""
    shape = ([50, 20], None, 4, 2, 128, True, 0)
    data = made(shape, "bfloat16", 8)
    all_of = both(shape, "bfloat16", data)
    q, k, v, w = (t.cuda() for t in data)
    s = starts_of([50, 20]).cuda()
    gq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    base = (view(w), view(q), view(k), view(v), view(all_of["out"]), view(all_of["log_sum"]))
    ocn.attention_grad(*base, view(gq), None, None, 1 / math.sqrt(128), view(s), view(s))
    ocn.attention_grad(*base, None, view(gk), view(gv), 1 / math.sqrt(128), view(s), view(s))
    ocn.attention_grad(*base, None, None, None, 1 / math.sqrt(128), view(s), view(s))
    assert torch.equal(gq, all_of["gq"]) and torch.equal(gk, all_of["gk"]) and torch.equal(gv, all_of["gv"])


def test_again_in_a_graph_and_over_a_capped_grid():
    """The same bits every time: eagerly, replayed with other work between, with two graphs that share a workspace, and in several launches"""
    from paper_1810_08723_amd import binding
    for shape in (([200, 60, 3], None, 8, 2, 128, True, 0), ([1, 2, 1], [1000, 40, 2000], 8, 2, 64, True, 0)):
        data = made(shape, "bfloat16", 9)
        first = both(shape, "bfloat16", data)
        binding.set_max_launch_blocks(3)
        try:
            again = both(shape, "bfloat16", data)
        finally:
            binding.set_max_launch_blocks(0)
        assert all(torch.equal(first[n], again[n]) for n in first)
        nq, nk, heads, kv, d, causal, window = shape
        q, k, v, w = (t.cuda() for t in data)
        s = [view(starts_of(x).cuda()) for x in (nq, nq if nk is None else nk)]
        need = max(ocn.attention_workspace_bytes(view(q), view(k), s[0]), ocn.attention_grad_workspace_bytes(view(q), view(k), s[0]))
        space = torch.empty(need, dtype=torch.uint8, device="cuda")
        graphs = []
        for _ in range(2):
            r = {n: torch.zeros_like(t) for n, t in first.items()}
            vr = {n: view(t) for n, t in r.items()}

            def call():
                ocn.attention(view(q), view(k), view(v), vr["out"], 1 / math.sqrt(d), *s, log_sum=vr["log_sum"], workspace=space)
                ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 1 / math.sqrt(d), *s, workspace=space)

            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                call()
            graphs.append((graph, r))
        for _ in range(3):
            for _, r in graphs:
                for t in r.values():
                    t.fill_(7)
            space.fill_(255)
            for graph, _ in graphs:
                graph.replay()
            both(shape, "bfloat16", data)
            for _, r in graphs:
                assert all(torch.equal(first[n], r[n]) for n in first)


def test_other_streams_at_once():
    shape = ([300, 100], None, 4, 2, 128, True, 0)
    data = made(shape, "half", 10)
    want = both(shape, "half", data)
    q, k, v, w = (t.cuda() for t in data)
    s = view(starts_of([300, 100]).cuda())
    runs = [{n: torch.zeros_like(t) for n, t in want.items()} for _ in range(3)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for stream, r in zip(streams, runs):
        vr = {n: view(t) for n, t in r.items()}
        ocn.attention(view(q), view(k), view(v), vr["out"], 1 / math.sqrt(128), s, s, log_sum=vr["log_sum"], stream=stream.cuda_stream)
        ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 1 / math.sqrt(128), s, s, stream=stream.cuda_stream)
    torch.cuda.synchronize()
    for r in runs:
        assert all(torch.equal(want[n], r[n]) for n in want)


@pytest.mark.parametrize("queries", [1, 40])
def test_offsets_past_32_bits(queries):
    """Keys and values that lie more than 4 GB apart"""
    nk, d = 70, 64
    far = torch.empty(nk * (1 << 26) + 1024, dtype=torch.uint8, device="cuda")
    k = torch.as_strided(far.view(torch.float16), (nk, 1, d), (1 << 25, d, 1))
    v = torch.as_strided(far.view(torch.float16), (nk, 1, d), (1 << 25, d, 1), 64)
    shape = ([queries], [nk], 4, 1, d, True, 0)
    data = made(shape, "half", 11)
    k.copy_(data[1])
    v.copy_(data[2])
    q, w = data[0].cuda(), data[3].cuda()
    s = [view(starts_of([n]).cuda()) for n in (queries, nk)]
    r = {"out": torch.zeros_like(q), "log_sum": torch.zeros(queries, 4, device="cuda"), "gq": torch.zeros_like(q), "gk": torch.zeros(nk, 1, d, dtype=torch.float16, device="cuda")}
    r["gv"] = torch.zeros_like(r["gk"])
    vr = {n: view(t) for n, t in r.items()}
    ocn.attention(view(q), view(k), view(v), vr["out"], 0.125, *s, log_sum=vr["log_sum"])
    ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 0.125, *s)
    check(shape, "half", data, r, 0.125)


def test_long_sequences_are_split_and_joined():
    """Single tokens over keys that many workgroups share; few sequences and many"""
    for lengths, heads, kv, d in (([9000], 4, 1, 64), ([1, 5000, 300], 8, 2, 128), ([700] * 20, 2, 1, 256)):
        for kind in KIND:
            shape = ([1] * len(lengths), lengths, heads, kv, d, True, 0)
            data = made(shape, kind, 12)
            check(shape, kind, data, both(shape, kind, data, grad=False))


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 40), (False, 0)])
def test_many_sequences(kind, causal, window):
    """More blocks than CUs, which are put in order: sequences of any lengths, ones without tokens among them"""
    g = torch.Generator().manual_seed(13)
    nq, nk = (torch.randint(0, 150, (90,), generator=g).tolist() for _ in range(2))
    for shape in ((nk, None, 8, 4, 64, causal, window), (nq, nk, 6, 6, 128, causal, window)):
        data = made(shape, kind, 14)
        check(shape, kind, data, both(shape, kind, data))


# few sequences of many rows, whose keys are cut into parts, and few keys of many rows, whose rows are; parts of which rows see none or some
SPLIT = [([600], [3001], 2, 1, 128, True, 0), ([200, 90], [1500, 40], 4, 2, 250, False, 0), ([700], None, 3, 1, 80, True, 300), ([1500, 64], [70, 64], 4, 2, 64, False, 0),
         ([900], [130], 6, 1, 128, True, 0), ([600], [300], 2, 2, 192, True, 100), ([333, 33], [1333, 1], 8, 8, 96, True, 700),
         ([2, 3], [3000, 700], 6, 2, 80, True, 0), ([1], [2500], 1, 1, 66, False, 0), ([400], [140], 5, 1, 77, True, 90)]


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("shape", SPLIT, ids=str)
def test_parts_of_long_sequences(shape, kind):
    from paper_1810_08723_amd import binding
    data = made(shape, kind, 15)
    got = both(shape, kind, data)
    check(shape, kind, data, got)
    binding.set_max_launch_blocks(7)
    try:
        again = both(shape, kind, data, how="packed")
    finally:
        binding.set_max_launch_blocks(0)
    assert all(torch.equal(got[n], again[n]) for n in got)


@pytest.mark.parametrize("kind", list(KIND))
def test_parts_with_odd_values_and_large_ones(kind):
    """Keys past 2900 are NaNs and infinities, which the rows that do not see them do without; a key of one part whose scores are far above all others"""
    shape = ([600], [3001], 2, 1, 128, True, 0)
    data = made(shape, kind, 16)
    q, k, v, w = (t.clone() for t in data)
    k[100] *= 20
    ref = reference(shape, kind, (q, k, v, w), grad=False)
    k[2950], v[2901], v[2990] = math.nan, math.inf, -math.inf
    got = both(shape, kind, (q, k, v, w), grad=False)
    clean = torch.arange(600) <= 2900 - 2401          # row i sees the keys up to i + 2401
    for n, bound_kind in (("out", kind), ("log_sum", None)):
        close(n, got[n][clean.cuda()], tuple(x[clean] for x in ref[n]), bound_kind)
    assert not got["out"][~clean.cuda()].isfinite().all(-1).any()


@pytest.mark.parametrize("size", [1e-4, 1.0, 1e4])
def test_parts_of_gradients_of_any_size_in_half(size):
    """Rows whose gradients differ by 2^20 from part to part: each part has a range of its own"""
    shape = ([1200], [100], 2, 1, 64, False, 0)
    q, k, v, w = made(shape, "half", 17)
    w = (w.float().clamp(-2, 2) * size * torch.logspace(0, -6, 1200)[:, None, None]).half()
    data = (q, k, v, w)
    got = both(shape, "half", data)
    want = reference(shape, "half", data, None, got["out"].cpu())
    for n in ("gq", "gk", "gv"):
        value, bound = want[n]
        fine = value.abs() < 65000
        close(n, torch.where(fine.cuda(), got[n], 0), tuple(torch.where(fine, x, 0.0) for x in (value, bound)), "half")


@pytest.mark.parametrize("kind", list(KIND))
def test_sequences_as_a_dimension_with_a_window(kind):
    """[batch, tokens, heads, channels] with more keys than queries, transposed and broadcast operands; the results of the same sequences packed"""
    batch, n, m, heads, kv, d = 3, 40, 75, 4, 2, 72
    g = torch.Generator().manual_seed(18)
    q, k, v, w = (torch.randn(batch, h, t, d, generator=g).to(KIND[kind]).cuda().transpose(1, 2) for h, t in ((heads, n), (kv, m), (kv, m), (heads, n)))
    k = k[:1].expand(batch, -1, -1, -1)
    for causal, window in ((True, 30), (False, 0)):
        r = {"out": torch.zeros_like(q), "log_sum": torch.zeros(batch, n, heads, device="cuda"), "gq": torch.zeros_like(q), "gk": torch.zeros(k.shape, dtype=k.dtype, device="cuda"), "gv": torch.zeros_like(v)}
        vr = {name: view(t) for name, t in r.items()}
        ocn.attention(view(q), view(k), view(v), vr["out"], 0.1, causal=causal, window=window, log_sum=vr["log_sum"])
        ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 0.1, causal=causal, window=window)
        shape = ([n] * batch, [m] * batch, heads, kv, d, causal, window)
        data = tuple(t.flatten(0, 1).cpu() for t in (q, k, v, w))
        check(shape, kind, data, {name: t.flatten(0, 1) for name, t in r.items()}, 0.1)


@pytest.mark.parametrize("kind", list(KIND))
@pytest.mark.parametrize("window", [19, 20, 2 ** 31 - 1, 2 ** 31, 2 ** 62])
def test_windows_of_all_keys_and_more(kind, window):
    """With more queries than keys, too, where positions relative to the keys are negative; the bits of no window"""
    shape = ([50, 300, 20], [20, 7, 20], 4, 2, 64, True, window)
    data = made(shape, kind, 19)
    got = both(shape, kind, data)
    check(shape, kind, data, got)
    if window > 19:
        want = both(shape[:6] + (0,), kind, data)
        assert all(torch.equal(got[n], want[n]) for n in got)


@pytest.mark.parametrize("kind", list(KIND))
def test_nothing_of_something(kind):
    """No queries, keys, heads, channels, sequences: zeros where there is somewhere to put them"""
    for tokens, keys, heads, kv, d in ((0, 9, 4, 2, 64), (9, 0, 4, 2, 64), (0, 0, 4, 2, 64), (9, 9, 0, 2, 64), (9, 9, 0, 0, 64), (9, 9, 4, 2, 0), (9, 9, 4, 2, 1)):
        q, k = torch.randn(tokens, heads, d), torch.randn(keys, kv, d)
        data = tuple(t.to(KIND[kind]) for t in (q, k, torch.randn_like(k), torch.randn_like(q)))
        shape = ([tokens], [keys], heads, kv, d, True, 0)
        got = both(shape, kind, data, 0.3)
        assert all((got[n] == 0).all() for n in ("gq", "gk", "gv") if tokens == 0 or keys == 0 or heads == 0), (tokens, keys, heads, kv, d)
        if d == 0:
            want = torch.arange(1, 10).double().log()[:, None]          # every score is zero
            assert ((got["log_sum"].double().cpu() - want).abs() <= 4 * 2.0 ** -24 * (1 + want)).all()
        elif keys == 0:
            assert (got["out"] == 0).all() and (got["log_sum"] == -math.inf).all()
        elif d == 1:
            check(shape, kind, data, got, 0.3)
        # sequences of nothing at all, as a dimension
        ocn.attention(*(view(torch.zeros(0, n, h, d, dtype=KIND[kind], device="cuda")) for n, h in ((tokens, heads), (keys, kv), (keys, kv), (tokens, heads))), 0.3)


def test_the_same_tensor_as_all_operands():
    """Queries, keys, values and the gradient of the results may be one tensor"""
    for kind in KIND:
        shape = ([70, 9], None, 2, 2, 64, True, 0)
        x = made(shape, kind, 20)[0]
        want = both(shape, kind, (x, x.clone(), x.clone(), x.clone()))
        check(shape, kind, (x, x, x, x), want)
        t = x.cuda()
        v, s = view(t), view(starts_of([70, 9]).cuda())
        r = {n: torch.zeros_like(y) for n, y in want.items()}
        vr = {n: view(y) for n, y in r.items()}
        ocn.attention(v, v, v, vr["out"], 0.125, s, s, log_sum=vr["log_sum"])
        ocn.attention_grad(v, v, v, v, vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 0.125, s, s)
        assert all(torch.equal(r[n], want[n]) for n in want)


@pytest.mark.parametrize("tokens,keys", [(300, 300), (6, 900)])
def test_a_replayed_graph_follows_its_starts(tokens, keys):
    """Lengths that change between replays: few and many rows, empty sequences, one of all tokens, tokens of none"""
    heads, kv, d = 4, 2, 64
    data = made(([tokens], [keys], heads, kv, d, True, 0), "bfloat16", 21)
    q, k, v, w = (t.cuda() for t in data)
    starts = [torch.zeros(5, dtype=torch.int32, device="cuda") for _ in range(2)]
    r = {"out": torch.zeros_like(q), "log_sum": torch.zeros(q.shape[:2], device="cuda"), "gq": torch.zeros_like(q), "gk": torch.zeros_like(k), "gv": torch.zeros_like(v)}
    vr, s = {n: view(t) for n, t in r.items()}, [view(t) for t in starts]

    def call():
        ocn.attention(view(q), view(k), view(v), vr["out"], 0.125, *s, log_sum=vr["log_sum"])
        ocn.attention_grad(view(w), view(q), view(k), view(v), vr["out"], vr["log_sum"], vr["gq"], vr["gk"], vr["gv"], 0.125, *s)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for part in ([0, 0.2, 0.2, 0.9, 1], [0, 0, 0, 0, 1], [0.1, 0.5, 0.6, 0.6, 0.7], [1, 1, 1, 1, 1], [0, 0.3, 0.4, 0.8, 1]):
        for t, n in zip(starts, (tokens, keys)):
            t.copy_(torch.tensor([int(x * n) for x in part], dtype=torch.int32))
        for t in r.values():
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in r.items()}
        sq, sk = spans(starts[0].cpu(), tokens), spans(starts[1].cpu(), keys)
        want = attended(*(t.cpu() for t in (q, k, v)), sq, sk, 0.125, True, 0, "bfloat16", w.cpu(), got["out"].cpu())
        for n in got:
            close(n, got[n], want[n], None if n == "log_sum" else "bfloat16")
            assert (got[n].cpu()[want[n][0].isnan()] == 7.0).all()
        call()
        assert all(torch.equal(got[n], r[n]) for n in got)


def test_one_buffer_of_queries_keys_and_values_and_one_of_their_gradients():
    shape = ([90, 1, 40], None, 4, 2, 64, True, 0)
    data = made(shape, "half", 22)
    want = both(shape, "half", data)
    x, g = (torch.full((131, 8, 64), 7.0, dtype=torch.float16, device="cuda") for _ in range(2))
    for t, part in zip(x.split([4, 2, 2], 1), data[:3]):
        t.copy_(part)
    q, k, v = (view(t) for t in x.split([4, 2, 2], 1))
    gq, gk, gv = (view(t) for t in g.split([4, 2, 2], 1))
    out, log, s = torch.zeros_like(want["out"]), torch.zeros_like(want["log_sum"]), view(starts_of(shape[0]).cuda())
    ocn.attention(q, k, v, view(out), 0.125, s, s, log_sum=view(log))
    ocn.attention_grad(view(data[3].cuda()), q, k, v, view(out), view(log), gq, gk, gv, 0.125, s, s)
    assert torch.equal(out, want["out"]) and torch.equal(log, want["log_sum"])
    assert torch.equal(g, torch.cat([want["gq"], want["gk"], want["gv"]], 1))


def test_more_sequences_than_are_put_in_order():
    """2600 short sequences, some of them empty"""
    lengths = torch.randint(0, 9, (2600,), generator=torch.Generator().manual_seed(23)).tolist()
    shape = (lengths, None, 1, 1, 16, True, 0)
    data = made(shape, "half", 23)
    check(shape, "half", data, both(shape, "half", data))
