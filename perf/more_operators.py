"""A layer's operators in training and over whole prompts, measured: attention over packed sequences, forward and with its
gradient, rotary positions with several axes, and the layer norm with its gradient.

`run` computes them in plain torch operations, or, where `own` is true, through the framework's public calls.  A case is
a dict of plain values; "op" says which operator it is, `_KEYS` below what the others mean.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda"
TYPES = {"half": torch.float16, "bfloat16": torch.bfloat16, "float": torch.float32}
SIZE = {"half": 2, "bfloat16": 2, "float": 4}
EPS = 1e-5
PADDED = 1 << 26     # scores up to which the plain form takes all sequences at once, padded to the longest
PIECE = 1 << 32      # ... that it holds at a time at most

_KEYS = """
type: of the inputs and outputs; heads, kv_heads, dim: query heads, heads of keys and values, channels of a head
attention, training (forward, then its gradient): sequences of shortest ... longest tokens, evenly spread, packed one behind the other;
  queries: the last so many tokens of each ask (0: all of them); causal; window: how far back a query sees (0: all)
axes: frames x rows x columns tokens, a position on each axis; rotary_dim: channels that rotate; shares: how the axes share the pairs ("row": one axis
  behind the other, "turn": in turn); interleaved: pairs (2i, 2i+1) rotate, else (i, i + rotary_dim/2); packed: the heads lie in one buffer
  [tokens, q heads + 2 * kv heads, dim]; inverse: the backward pass
layer: rows x width; offset: the mean of the inputs; weights: with weight and bias; grad: the backward pass
"""


def listed():
    attention = {"op": "attention", "type": "bfloat16", "batch": 1, "shortest": 64, "longest": 64, "queries": 0, "causal": True, "window": 0,
                 "heads": 32, "kv_heads": 8, "dim": 128}
    training = {**attention, "op": "training"}
    axes = {"op": "axes", "type": "bfloat16", "frames": 1, "rows": 1, "columns": 1, "heads": 32, "kv_heads": 8, "dim": 128, "rotary_dim": 128,
            "shares": "row", "interleaved": False, "packed": True, "inverse": False}
    layer = {"op": "layer", "type": "bfloat16", "rows": 48, "width": 4096, "offset": 0.0, "weights": True, "grad": False}
    return [
        # a few short prompts, packed: latency
        {**attention, "name": "attention: short prompts", "batch": 5, "shortest": 9, "longest": 61},
        # prompts of a serving batch, of very different lengths
        {**attention, "name": "attention: prompts", "batch": 16, "shortest": 101, "longest": 6000},
        # one long document
        {**attention, "name": "attention: long", "type": "half", "shortest": 30011, "longest": 30011, "heads": 16, "kv_heads": 4, "dim": 64},
        # the next token of each of 48 sequences, over keys and values as they are
        {**attention, "name": "attention: next tokens", "type": "half", "batch": 48, "shortest": 1, "longest": 8192, "queries": 1},
        # a training step on two short texts: latency
        {**training, "name": "training: short", "batch": 2, "shortest": 130, "longest": 130, "heads": 8, "kv_heads": 8, "dim": 64},
        # a training batch
        {**training, "name": "training: batch", "batch": 4, "shortest": 4096, "longest": 4096},
        # images of different sizes in training: all patches see each other
        {**training, "name": "training: images", "type": "half", "batch": 9, "shortest": 77, "longest": 2903, "causal": False, "heads": 16,
         "kv_heads": 16, "dim": 80},
        # the queries of one generated token: latency
        {**axes, "name": "axes: one token"},
        # the queries of a video's patches, an odd number of them
        {**axes, "name": "axes: video", "frames": 9, "rows": 45, "columns": 61},
        # hidden states of a batch of generated tokens: latency
        {**layer, "name": "layer norm: 48 tokens"},
        # hidden states of images' patches, far from zero
        {**layer, "name": "layer norm: patches", "type": "half", "rows": 24705, "width": 1280, "offset": 3.0},
        # a training step's backward pass, weights and biases with it
        {**layer, "name": "layer norm: gradient", "rows": 16384, "grad": True},
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attention", "training", "axes", "layer"))
    c = {"op": op, "type": rng.choice(("half", "bfloat16", "bfloat16", "float"))}
    if op == "layer":
        c["width"] = rng.choice((_spread(rng, 33, 16384), 8 * _spread(rng, 16, 1024)))
        c["rows"] = rng.choice((_spread(rng, 1, 300), _spread(rng, 300, 6 * 10**7 // c["width"] + 300)))
        c["offset"] = rng.choice((0.0, 0.0, rng.uniform(-8.0, 8.0)))
        c["weights"] = rng.random() < 0.8
        c["grad"] = rng.random() < 0.5
        return c
    kv = rng.choice((1, 2, 4, 8))
    c["kv_heads"], c["heads"] = kv, kv * rng.choice((1, 2, 3, 4, 7, 8))
    if op == "axes":
        c["dim"] = rng.choice((64, 80, 96, 128, 128, 160, 256))
        c["rotary_dim"] = rng.choice((c["dim"], c["dim"], c["dim"] // 2))
        c["shares"] = rng.choice(("row", "row", "turn"))
        c["interleaved"], c["packed"], c["inverse"] = (rng.random() < 0.4 for _ in range(3))
        tokens = _spread(rng, 1, 64 * 10**6 // ((c["heads"] + 2 * kv) * c["dim"]))
        c["frames"] = rng.choice((1, _spread(rng, 1, 16)))
        c["rows"] = max(1, int(math.sqrt(tokens / c["frames"] * rng.uniform(0.3, 1.0))))
        c["columns"] = max(1, tokens // (c["frames"] * c["rows"]))
        return c
    c["dim"] = rng.choice((64, 64, 80, 96, 128, 128, 128, 256, rng.randint(17, 250)))
    c["batch"] = _spread(rng, 1, 48)
    c["queries"] = rng.choice((0, 0, 1, _spread(rng, 2, 500))) if op == "attention" else 0
    c["causal"] = c["queries"] != 0 or rng.random() < 0.75
    # scores times channels: what the largest listed case has, less for float and for gradients
    most = 4.0e11 / (1 if c["type"] != "float" else 4) / (1 if op == "attention" else 3.5) / (c["batch"] * c["heads"] * c["dim"])
    top = int(math.sqrt(most)) if not c["queries"] else int(min(most / c["queries"], 4 * 10**8 / (c["batch"] * kv * c["dim"])))
    c["longest"] = _spread(rng, 24, max(32, min(32768, top)))
    c["shortest"] = rng.choice((c["longest"], rng.randint(0, c["longest"])))
    c["window"] = rng.choice((0, 0, 0, _spread(rng, 8, 4096))) if c["causal"] else 0
    return c


# ---- what the cases are made of ---------------------------------------------------------------


def _lengths(case):
    """Tokens of each sequence"""
    lo, hi, n = case["shortest"], case["longest"], case["batch"]
    return [hi] if n == 1 else [lo + (hi - lo) * i // (n - 1) for i in range(n)]


def _asking(case):
    """... and queries"""
    return [case["queries"] or n for n in _lengths(case)]


def _pairs(nq, nk, causal, window):
    """How many pairs of a query and a key there are"""
    if not causal:
        return nq * nk
    def up_to(n):       # 1 + 2 + ... + n, nothing for n < 1
        return n * (n + 1) // 2 if n > 0 else 0
    pairs = up_to(nk) - up_to(nk - nq)
    return pairs - (up_to(nk - window) - up_to(nk - window - nq) if window else 0)


def work(case):
    size = SIZE[case["type"]]
    if case["op"] == "layer":
        n = case["rows"] * case["width"]
        return {"bytes": (3 if case["grad"] else 2) * n * size, "flops": (14.0 if case["grad"] else 8.0) * n}
    if case["op"] == "axes":
        n = case["frames"] * case["rows"] * case["columns"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size, "flops": 3.0 * n}
    keys, queries, d = _lengths(case), _asking(case), case["dim"]
    pairs = sum(_pairs(q, k, case["causal"], case["window"]) for q, k in zip(queries, keys))
    held = [min(k, case["window"] + q) if case["window"] else k for q, k in zip(queries, keys)]
    once = 2 * (sum(queries) * case["heads"] + sum(held) * case["kv_heads"]) * d * size
    if case["op"] == "attention":
        return {"bytes": once, "flops": 4.0 * pairs * case["heads"] * d}
    return {"bytes": 2 * once, "flops": 14.0 * pairs * case["heads"] * d}


def _shares(case):
    """The axis of each pair"""
    pairs = case["rotary_dim"] // 2
    if case["shares"] == "turn":
        return [i % 3 for i in range(pairs)]
    first = pairs - 2 * (pairs // 3)
    return [0 if i < first else 1 if i < first + pairs // 3 else 2 for i in range(pairs)]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    op, kind = case["op"], TYPES[case["type"]]
    s = {"case": case, "op": op}

    def normal(*shape):
        return torch.randn(shape, device=DEVICE, generator=gen)

    if op == "layer":
        rows, width = case["rows"], case["width"]
        s["x"] = (normal(rows, width) * (0.5 + normal(rows, 1).abs()) + case["offset"]).to(kind)
        s["weight"], s["bias"] = ((1.0 + 0.2 * normal(width)).to(kind), (0.2 * normal(width)).to(kind)) if case["weights"] else (None, None)
        s["out"] = torch.empty_like(s["x"])
        names = ["x", "out"] + (["weight", "bias"] if case["weights"] else [])
        if case["grad"]:
            s["gout"] = normal(rows, width).to(kind)
            if case["weights"]:
                s["gweight"], s["gbias"] = (torch.empty(width, dtype=torch.float32, device=DEVICE) for _ in range(2))
            names += ["gout"] + (["gweight", "gbias"] if case["weights"] else [])
    elif op == "axes":
        tokens, h = case["frames"] * case["rows"] * case["columns"], case["heads"]
        all_heads = h + 2 * case["kv_heads"] if case["packed"] else h
        s["x"] = normal(tokens, all_heads, case["dim"]).to(kind)[:, :h]
        s["out"] = torch.empty(tokens, h, case["dim"], dtype=kind, device=DEVICE)
        # where the picture begins in its text, then frame, row and column
        first = torch.randint(0, 100000, (1,), device=DEVICE, generator=gen)
        grid = torch.meshgrid(*(torch.arange(n, device=DEVICE) for n in (case["frames"], case["rows"], case["columns"])), indexing="ij")
        s["positions"] = (first + torch.stack([g.reshape(-1) for g in grid])).to(torch.int32)
        s["axis"] = torch.tensor(_shares(case), device=DEVICE)
        pair = torch.arange(case["rotary_dim"] // 2, dtype=torch.float64, device=DEVICE)
        s["frequencies"] = 10000.0 ** (-2.0 * pair / case["rotary_dim"])
        names = ["x", "out", "positions"]
    else:
        keys, queries = _lengths(case), _asking(case)
        s["k_starts"], s["q_starts"] = (torch.tensor([sum(n[:i]) for i in range(len(n) + 1)], dtype=torch.int32, device=DEVICE)
                                        for n in (keys, queries))
        h, kv, d = case["heads"], case["kv_heads"], case["dim"]
        s["q"] = (1.5 * normal(sum(queries), h, d)).to(kind)
        s["k"], s["v"] = (normal(sum(keys), kv, d).to(kind) for _ in range(2))
        s["scale"] = 1.0 / math.sqrt(d)
        s["out"] = torch.empty_like(s["q"])
        names = ["q", "k", "v", "out", "q_starts", "k_starts"]
        if op == "training":
            s["gout"] = normal(sum(queries), h, d).to(kind)
            s["gq"], s["gk"], s["gv"] = (torch.empty_like(s[n]) for n in "qkv")
            s["log_sum"] = torch.empty(sum(queries), h, dtype=torch.float32, device=DEVICE)
            names += ["gout", "gq", "gk", "gv", "log_sum"]
    if own:      # the descriptors, the rotation and the workspace that a program keeps beside its buffers
        ocn = _framework()
        v = s["views"] = {n: _view(s[n]) for n in names}
        need = 0
        if op == "axes":
            pairs = case["rotary_dim"] // 2
            table = ocn.rotary_axes([_shares(case).count(a) for a in range(3)], [10000.0 ** (-2.0 * i / case["rotary_dim"]) for i in range(pairs)],
                                    case["shares"])
            s["table"] = torch.tensor(table, dtype=torch.float64, device=DEVICE)
            s["rotation"] = ocn.Rotation(v["positions"], _view(s["table"]), case["rotary_dim"], "interleaved" if case["interleaved"] else "half")
        elif op == "layer":
            need = ocn.layer_norm_grad_workspace_bytes(v["x"]) if case["grad"] else 0
        else:
            need = ocn.attention_workspace_bytes(v["q"], v["k"], v["q_starts"])
            if op == "training":
                need = max(need, ocn.attention_grad_workspace_bytes(v["q"], v["k"], v["q_starts"]))
        s["workspace"] = torch.empty(max(1, need), dtype=torch.uint8, device=DEVICE)
    return s


# ---- the framework's calls -------------------------------------------------------------------------


def _framework():
    import paper_1810_08723_amd as ocn
    return ocn


_NAMES = {torch.float16: "half", torch.bfloat16: "bfloat16", torch.float32: "float", torch.float64: "double", torch.int32: "int32"}


def _view(t):
    e = t.element_size()
    return _framework().Tensor(t.data_ptr(), _NAMES[t.dtype], tuple(t.shape), tuple(n * e for n in t.stride()), 0, t.device.index or 0, t)


def _run_own(s):
    ocn, c, v = _framework(), s["case"], s["views"]
    if s["op"] == "axes":
        ocn.rotary(v["x"], s["rotation"], v["out"], inverse=c["inverse"])
        return s["out"]
    if s["op"] == "layer":
        if not c["grad"]:
            ocn.layer_norm(v["x"], v.get("weight"), v.get("bias"), v["out"], eps=EPS)
            return s["out"]
        ocn.layer_norm_grad(v["gout"], v["x"], v.get("weight"), v["out"], v.get("gweight"), v.get("gbias"), eps=EPS, workspace=s["workspace"])
        return [s["out"]] + ([s["gweight"], s["gbias"]] if c["weights"] else [])
    how = {"q_starts": v["q_starts"], "k_starts": v["k_starts"], "causal": c["causal"], "window": c["window"], "workspace": s["workspace"]}
    ocn.attention(v["q"], v["k"], v["v"], v["out"], s["scale"], log_sum=v.get("log_sum"), **how)
    if s["op"] == "attention":
        return s["out"]
    ocn.attention_grad(v["gout"], v["q"], v["k"], v["v"], v["out"], v["log_sum"], v["gq"], v["gk"], v["gv"], s["scale"], **how)
    return [s["out"], s["gq"], s["gk"], s["gv"]]


# ---- the plain forms: elementary operations in 32 bits, angles and long sums in 64 ------------------------


def _layer(s):
    c = s["case"]
    x = s["x"].float()
    x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    unit = x * r
    w = s["weight"].float() if c["weights"] else None
    if not c["grad"]:
        return (unit * w + s["bias"].float() if c["weights"] else unit).to(s["x"].dtype)
    g = s["gout"].float()
    gw = g * w if c["weights"] else g
    gx = (r * (gw - gw.mean(-1, keepdim=True) - unit * (gw * unit).mean(-1, keepdim=True))).to(s["x"].dtype)
    return [gx] + ([(g * unit).double().sum(0).float(), g.double().sum(0).float()] if c["weights"] else [])


def _axes(s):
    c = s["case"]
    r = c["rotary_dim"]
    angle = s["positions"].double()[s["axis"]].t() * s["frequencies"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if c["inverse"]:
        sin = -sin
    x = s["x"].float()
    out = x.clone()
    one, two = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., one], x[..., two]
    out[..., one] = a * cos - b * sin
    out[..., two] = b * cos + a * sin
    return out.to(s["x"].dtype)


def _pieces(case):
    """What is computed at a time: sequences, and heads of keys and values.  All at once, padded to the longest, where that is little; else
    a sequence at a time, with as many heads as there is room for."""
    keys, queries, kv = _lengths(case), _asking(case), case["kv_heads"]
    if len(keys) * case["heads"] * max(keys) * max(queries) <= PADDED:
        return [(list(range(len(keys))), 0, kv)]
    per = [max(1, min(kv, PIECE // max(1, k * q * case["heads"] // kv))) for k, q in zip(keys, queries)]
    return [([i], h, min(kv, h + per[i])) for i in range(len(keys)) for h in range(0, kv, per[i])]


def _places(starts, which, longest, rows):
    """Rows [sequences, longest] of a packed tensor; past a sequence's end: `rows`"""
    first, end = starts[which[0]:which[-1] + 1, None], starts[which[0] + 1:which[-1] + 2, None]
    at = first + torch.arange(longest, device=DEVICE)
    return torch.where(at < end, at, rows).long()


def _attention(s):
    c = s["case"]
    keys, queries = _lengths(c), _asking(c)
    h, kv, d = c["heads"], c["kv_heads"], c["dim"]
    per = h // kv
    tq, tk = sum(queries), sum(keys)
    grad = s["op"] == "training"
    out = torch.zeros(tq + 1, kv, per, d, device=DEVICE)       # (the row behind the last takes what is padded)
    gq = torch.zeros_like(out) if grad else None
    gk, gv = (torch.zeros(tk + 1, kv, d, device=DEVICE) if grad else None for _ in range(2))
    for which, lo, hi in _pieces(c):
        nq, nk = max(queries[i] for i in which), max(keys[i] for i in which)
        if nq == 0 or nk == 0:
            continue
        at_q, at_k = _places(s["q_starts"], which, nq, tq), _places(s["k_starts"], which, nk, tk)

        def rows(x):       # [sequences, kv heads, queries * heads to a kv head, dim]
            x = x.view(tq, kv, per, d)[at_q.clamp(max=tq - 1), lo:hi].float()
            return x.permute(0, 2, 1, 3, 4).reshape(len(which), hi - lo, nq * per, d)

        def columns(x):    # [sequences, kv heads, keys, dim]
            return x[at_k.clamp(max=tk - 1), lo:hi].float().permute(0, 2, 1, 3).contiguous()

        def back(x):
            return x.view(len(which), hi - lo, nq, per, d).permute(0, 2, 1, 3, 4)

        q, k, v = rows(s["q"]), columns(s["k"]), columns(s["v"])
        score = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(s["scale"])
        lengths = [(s[n][which[0] + 1:which[-1] + 2] - s[n][which[0]:which[-1] + 1])[:, None, None] for n in ("q_starts", "k_starts")]
        j = torch.arange(nk, device=DEVICE)
        hidden = j >= lengths[1]
        if c["causal"]:
            last = torch.arange(nq, device=DEVICE).repeat_interleave(per)[:, None] + (lengths[1] - lengths[0])
            hidden = hidden | (j > last)
            if c["window"]:
                hidden = hidden | (j <= last - c["window"])
        score.masked_fill_(hidden[:, None], -math.inf)
        top = score.amax(-1, keepdim=True)
        p = score.sub_(torch.where(top > -math.inf, top, torch.zeros_like(top))).exp_()
        total = p.sum(-1, keepdim=True)
        p.div_(torch.where(total > 0, total, torch.ones_like(total)))
        o = torch.matmul(p, v)
        out[at_q, lo:hi] = back(o)
        if grad:
            g = rows(s["gout"])
            g = g.masked_fill((at_q == tq).repeat_interleave(per, 1)[:, None, :, None], 0.0)
            gv[at_k, lo:hi] = torch.matmul(p.transpose(-1, -2).contiguous(), g).permute(0, 2, 1, 3)
            gs = torch.matmul(g, v.transpose(-1, -2).contiguous()).sub_((g * o).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
            del p, score
            gq[at_q, lo:hi] = back(torch.matmul(gs, k))
            gk[at_k, lo:hi] = torch.matmul(gs.transpose(-1, -2).contiguous(), q).permute(0, 2, 1, 3)
    kind = s["q"].dtype
    out = out[:tq].reshape(tq, h, d).to(kind)
    return [out, gq[:tq].reshape(tq, h, d).to(kind), gk[:tk].to(kind), gv[:tk].to(kind)] if grad else out


def run(s):
    if own:
        return _run_own(s)
    return _layer(s) if s["op"] == "layer" else _axes(s) if s["op"] == "axes" else _attention(s)


# ---- the definitions in 64 bits, apart from the forms above ------------------------------------------


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    if s["op"] == "layer":
        x = s["x"].double()
        n = case["width"]
        mean = x.sum(1) / n
        deviation = ((x - mean[:, None]).square().sum(1) / n + EPS).sqrt()
        unit = (x - mean[:, None]) / deviation[:, None]
        w, b = (s[m].double() if case["weights"] else torch.full((), f, dtype=torch.float64, device=DEVICE) for m, f in (("weight", 1.0), ("bias", 0.0)))
        if not case["grad"]:
            return torch.addcmul(b.expand(n), unit, w.expand(n))
        g = s["gout"].double()
        # the gradient through the projections that the norm is: off the ones, and off the unit row
        h = g * w
        h = h - h.sum(1, keepdim=True) / n
        h = h - unit * ((h * unit).sum(1, keepdim=True) / n)
        return [h / deviation[:, None]] + ([(unit * g).sum(0), g.sum(0)] if case["weights"] else [])
    if s["op"] == "axes":
        r = case["rotary_dim"]
        x = s["x"].double()
        which = _shares(case)
        turn = torch.ones(x.shape[0], r // 2, dtype=torch.complex128, device=DEVICE)
        for a in range(3):         # a turn for each axis, of the pairs that are its own
            mine = torch.tensor([n == a for n in which], device=DEVICE)
            angle = torch.outer(s["positions"][a].double(), s["frequencies"]) * mine
            turn = turn * torch.complex(angle.cos(), -angle.sin() if case["inverse"] else angle.sin())
        pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn[:, None])
        z = z.flatten(-2) if case["interleaved"] else z.transpose(-1, -2).flatten(-2)
        return torch.cat([z, x[..., r:]], -1)
    grad = s["op"] == "training"
    per = case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    gq = torch.zeros_like(out)
    gk, gv = (torch.zeros(s["k"].shape, dtype=torch.float64, device=DEVICE) for _ in range(2))
    q_at = k_at = 0
    for nq, nk in zip(_asking(case), _lengths(case)):
        block = max(1, min(nq, (1 << 28) // max(1, nk * per)))
        for a in range(case["kv_heads"] if nk else 0):
            keys = slice(k_at, k_at + nk)
            k, v = s["k"][keys, a].double(), s["v"][keys, a].double()
            kt, vt = k.t().contiguous(), v.t().contiguous()
            for at in range(0, nq, block):      # some queries, each with its first and last key
                n = min(block, nq - at)
                rows, heads = slice(q_at + at, q_at + at + n), slice(a * per, (a + 1) * per)
                last = torch.arange(at, at + n, device=DEVICE) + (nk - nq) if case["causal"] else torch.full((n,), nk - 1, device=DEVICE)
                first = last - case["window"] + 1 if case["window"] else torch.zeros_like(last)
                q = s["q"][rows, heads].double().reshape(n * per, -1)
                logit = (q @ kt * s["scale"]).view(n, per, nk)
                j = torch.arange(nk, device=DEVICE)
                sees = ((j <= last[:, None]) & (j >= first[:, None]))[:, None]
                logit = logit.masked_fill_(~sees, -math.inf)
                log_sum = torch.logsumexp(logit, -1, keepdim=True)
                p = logit.sub_(log_sum.masked_fill(log_sum == -math.inf, 0.0)).exp_().view(n * per, nk)
                o = p @ v
                out[rows, heads] = o.view(n, per, -1)
                if not grad:
                    continue
                g = s["gout"][rows, heads].double().reshape(n * per, -1)
                gv[keys, a] += p.t().contiguous() @ g
                gp = g @ vt
                gs = (gp - (gp * p).sum(1, keepdim=True)) * p * s["scale"]
                gq[rows, heads] = (gs @ k).view(n, per, -1)
                gk[keys, a] += gs.t().contiguous() @ q
        q_at, k_at = q_at + nq, k_at + nk
    return [out, gq, gk, gv] if grad else out
