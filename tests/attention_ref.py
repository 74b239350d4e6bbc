"""Attention over whole sequences and its gradient in 64 bits on the CPU, with how far the framework's results may be from it.

Bounds.  u = 2^-24 is half a step of single precision, t half a step of the tensors' type (0 where products are taken in single precision throughout: float).
    score        a sum of d products: off by (d + 2) u sum|q k| |scale| =: a; two such differ from their maximum's by 2 a, and the exponential and its argument add
                 4 u (1 + |score - best|)
    weight       p off by e = exp(2 a + ...) - 1 of itself before it is rounded, by t more after; a half that is below 2^-14 by 2^-25: the reference's weight is 2^9 and a row's sum is
                 as much or more, so that this is 2^-34 of the sum; in the gradient 1 is 2^12, so that it is 2^-37, and the largest s of a column so far 2^11 or more, 2^-36 of that
    out          the product with v is a sum of n terms and the sum of weights as well: (2 n + 16) u, all of it times sum p |v|
    log_sum      a + (n + 16) u, and 4 u of itself
    gradient     the weight is made again from log_sum, which is off as above;  gout v off by (d + 2) u sum|gout v|;  gout out by what out is, and (d + 2) u;
                 s = p (gout v - gout out) has the errors of both and is rounded (t);  sums of n terms, n u
"""
import torch

from heads_ref import F32, half_step


def spans(starts, tokens):
    at = [min(max(int(x), 0), tokens) for x in starts]
    return [(a, max(a, b)) for a, b in zip(at, at[1:])]


def seen(n, m, causal, window):
    """[n queries, m keys]"""
    i, j = torch.arange(n)[:, None], torch.arange(m)[None]
    s = torch.ones(n, m, dtype=torch.bool)
    if causal:
        s &= j <= i + m - n
        if window:
            s &= j > i + m - n - window
    return s


def attended(q, k, v, q_spans, k_spans, scale, causal, window, kind, gout=None, kept=None):
    """q [tokens, heads, d], k and v [keys, kv, d] (any type).  A dict of (value, bound): out, log_sum, and with gout: gq, gk, gv; rows of no sequence are NaN.
    `kept`: the out that the gradient is given, in its type"""
    qd, kd, vd = q.double(), k.double(), v.double()
    heads, kv, d = q.shape[1], k.shape[1], q.shape[2]
    u, t = F32, (0.0 if kind == "float" else half_step(kind))
    tiny = 2.0 ** -36 if kind == "half" else 0.0            # of s and (more than) of p in the gradient; of weights 4 times that
    r = {"out": torch.full_like(qd, float("nan")), "log_sum": torch.full(q.shape[:2], float("nan"), dtype=torch.float64)}
    b = {n: x.clone() for n, x in r.items()}
    if gout is not None:
        gd = gout.double()
        for n, x in (("gq", qd), ("gk", kd), ("gv", vd)):
            r[n], b[n] = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    for (q0, q1), (k0, k1) in zip(q_spans, k_spans):
        n, m = q1 - q0, k1 - k0
        see = seen(n, m, causal, window)
        if gout is not None:
            for name in ("gk", "gv"):
                r[name][k0:k1], b[name][k0:k1] = 0.0, 0.0
        for h in range(heads):
            g = h * kv // heads
            x, y, z = qd[q0:q1, h], kd[k0:k1, g], vd[k0:k1, g]
            s = (x @ y.t() * scale).masked_fill(~see, -float("inf"))
            a = (x.abs() @ y.abs().t() * abs(scale) * (d + 2) * u).masked_fill(~see, 0.0)
            top = s.amax(1, keepdim=True) if m else torch.full((n, 1), -float("inf"), dtype=torch.float64)
            top = top.masked_fill(top == -float("inf"), 0.0)
            p = (s - top).exp()
            total = p.sum(1, keepdim=True)
            any_seen = total > 0
            p = torch.where(any_seen, p / total, 0.0)
            worst = a.amax(1, keepdim=True) if m else torch.zeros(n, 1, dtype=torch.float64)
            e = torch.expm1(a + worst + 4 * u * (1 + (s - top).abs().masked_fill(~see, 0.0)))
            out = p @ z
            size = p @ z.abs()
            off = (p * e) @ z.abs() + (p * e).sum(1, keepdim=True) * out.abs() + (t + (2 * m + 16) * u) * size + m * 4 * tiny * (z.abs().amax(0) if m else 0.0)
            r["out"][q0:q1, h], b["out"][q0:q1, h] = out, off
            log = torch.where(any_seen, total.log() + top, -float("inf"))
            log_off = worst + (p * e).sum(1, keepdim=True) + (m + 16) * u + 4 * u * torch.where(any_seen, log.abs() + top.abs(), 0.0)
            r["log_sum"][q0:q1, h], b["log_sum"][q0:q1, h] = log[:, 0], log_off[:, 0]
            if gout is None or m == 0 or n == 0:
                if gout is not None:
                    r["gq"][q0:q1, h], b["gq"][q0:q1, h] = 0.0, 0.0
                continue
            w = gd[q0:q1, h]
            dp, dp_off = w @ z.t(), w.abs() @ z.abs().t() * (d + 2) * u
            along = (w * out).sum(1, keepdim=True)
            o = out if kept is None else kept[q0:q1, h].double()
            along_off = (w * (o - out)).sum(1, keepdim=True).abs() + (d + 2) * u * (w * o).abs().sum(1, keepdim=True)
            c = p * (dp - along)
            pe = torch.expm1(a + log_off + 4 * u * (1 + torch.where(any_seen, log.abs(), 0.0) + (s - top).abs().masked_fill(~see, 0.0)))
            size = p * (dp.abs() + along.abs())
            c_off = p * (1 + pe) * (dp_off + along_off) + (pe + 4 * u) * size + t * c.abs() + t * p * (dp_off + along_off + pe * size)
            c_off = c_off + tiny * (c.abs().amax() + c_off.amax())
            p_off = p * (pe + t) + tiny
            gq = scale * (c @ y)
            r["gq"][q0:q1, h] = gq
            b["gq"][q0:q1, h] = abs(scale) * (c_off @ y.abs() + (m + 4) * u * (c.abs() @ y.abs()))
            r["gk"][k0:k1, g] += scale * (c.t() @ x)
            rows = n * heads // kv
            b["gk"][k0:k1, g] += abs(scale) * (c_off.t() @ x.abs() + (rows + 4) * u * (c.abs().t() @ x.abs()))
            r["gv"][k0:k1, g] += p.t() @ w
            b["gv"][k0:k1, g] += p_off.t() @ w.abs() + (rows + 4) * u * (p.t() @ w.abs())
    return {n: (r[n], b[n]) for n in r}
