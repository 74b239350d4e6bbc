"""Plain 64-bit forms of the operators over heads, on the CPU, and descriptors of torch tensors for them."""
import math

import numpy as np
import torch

import paper_1810_08723_amd as ocn

KIND = {"half": torch.float16, "bfloat16": torch.bfloat16, "float": torch.float32}
NAMES = {torch.float16: "half", torch.bfloat16: "bfloat16", torch.float32: "float", torch.float64: "double", torch.int32: "int32",
         torch.int64: "int64", torch.uint8: "uint8"}
UNITS = (0, 1, 2, 3, 4, 6, 8, 12)
F32 = 2.0 ** -24


def half_step(kind):
    return torch.finfo(KIND[kind]).eps / 2


def rounding(kind, want):
    """What rounding `want` to the type may change: half a step, those of subnormal numbers among them"""
    size = abs(want) * half_step(kind)
    least = {"half": 2.0 ** -25, "bfloat16": 2.0 ** -134, "float": 2.0 ** -150}[kind]
    return size.clamp(min=least) if isinstance(size, torch.Tensor) else np.maximum(size, least)


def view(t):
    e = t.element_size()
    return ocn.Tensor(t.data_ptr(), NAMES[t.dtype], tuple(t.shape), tuple(s * e for s in t.stride()), 0, t.device.index or 0, t)


def rotated(x, positions, frequencies, rotary_dim, interleaved=False, magnitude=1.0, back=False):
    """x [..., heads, channels] float64; positions broadcast against the leading dimensions.  Returns (rotated, |a| + |b| of each pair)"""
    angle = positions.double()[..., None] * frequencies.double()
    angle = angle.expand(*x.shape[:-2], rotary_dim // 2)[..., None, :]
    c, s = angle.cos() * magnitude, angle.sin() * magnitude * (-1 if back else 1)
    r = rotary_dim
    a, b = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    out, size = x.clone(), x.abs()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., b] * c + x[..., a] * s
    both = (x[..., a].abs() + x[..., b].abs()) * abs(magnitude)
    size[..., a] = both
    size[..., b] = both
    return out, size


def normed(x, w, eps):
    return x / (x.square().mean(-1, keepdim=True) + eps).sqrt() * w


def nine_bits(m):
    """float32 array to nine significant bits, ties to even, as float16"""
    b = np.asarray(m, np.float32).view(np.uint32).astype(np.uint64)
    b = ((b + 0x3fff + ((b >> 15) & 1)) & 0xffff8000).astype(np.uint32)
    return b.view(np.float32).astype(np.float16)


def held(x):
    """What the cache holds of x [..., channels] (float64 numpy, not rotated): values, by nearest distance, ties to the even code"""
    g = x.reshape(*x.shape[:-1], -1, 32)
    m = np.abs(g).max(-1).astype(np.float32)
    scale = nine_bits(np.minimum(m * np.float32(1 / 12), np.float32(5456))).astype(np.float64)[..., None]
    y = np.abs(g) / np.where(scale > 0, scale, 1)
    distance = np.abs(y[..., None] - np.array(UNITS))
    near = distance.min(-1, keepdims=True)
    tied = distance == near
    even = tied & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), tied.argmax(-1))
    code = np.where(scale > 0, code, 0)
    return (np.array(UNITS)[code] * scale * np.where(np.signbit(g), -1.0, 1.0)).reshape(x.shape)


def token_of_block(block, page, d, token):
    """(keys, values) of one token, float64 [channels], out of a block's bytes, place by place"""
    out = []
    for v in (False, True):
        row = np.empty(d)
        for c in range(d):
            if v:
                wide = d // 16
                at = page * d // 2 + ((token // 4 * 16 + c // wide) * 4 + token % 4) * (wide // 2) + c % wide // 2
            else:
                at = token * (d // 2) + c // 2
            code = int(block[at]) >> (4 * (c % 2)) & 15
            where = page * d + 2 * (((d // 32 if v else 0) + c // 32) * page + token)
            scale = float(block[where:where + 2].view(np.float16)[0])
            row[c] = (-1 if code & 8 else 1) * UNITS[code & 7] * scale
        out.append(row)
    return out


def values_of(cache, page, d):
    """(keys, values) of all blocks of [pages, heads, block] bytes (numpy): float64 [pages, heads, page, channels]"""
    lead = cache.shape[:-1]
    n = page * d // 2
    units = np.array(UNITS + tuple(-u for u in UNITS), np.float64)
    scales = np.ascontiguousarray(cache[..., 2 * n:]).view(np.float16).astype(np.float64).reshape(*lead, 2, d // 32, page)
    k = cache[..., :n].reshape(*lead, page, d // 2)
    v = cache[..., n:2 * n].reshape(*lead, page // 4, 16, 4, d // 32).swapaxes(-3, -2).reshape(*lead, page, d // 2)
    out = []
    for i, codes in enumerate((k, v)):
        x = np.stack([units[codes & 15], units[codes >> 4]], -1).reshape(*lead, page, d)
        out.append(x * np.repeat(scales[..., i, :, :].swapaxes(-1, -2), 32, axis=-1))
    return out


def attended(q, keys, values, table, seen, scale, window, page):
    """q [batch, queries, heads, channels] float64; keys, values of values_of().  Returns (out, log of the sum, sum p |v| / sum p,
    the largest sum |q k| * scale of a seen token) for each query head"""
    b, t, h, d = q.shape
    pages, kv = keys.shape[:2]
    out, size = np.zeros((b, t, h, d)), np.zeros((b, t, h, d))
    log, reach = np.full((b, t, h), -np.inf), np.zeros((b, t, h))
    for i in range(b):
        for j in range(t):
            n = min(int(seen[i, j]), table.shape[1] * page)
            tokens = [x for x in range(max(0, n - window) if window else 0, n) if 0 <= table[i, x // page] < pages]
            if not tokens:
                continue
            at = np.array(tokens)
            blocks = table[i, at // page]
            for m in range(h):
                k, v = keys[blocks, m * kv // h, at % page], values[blocks, m * kv // h, at % page]
                s = k @ q[i, j, m] * scale
                with np.errstate(invalid="ignore"):
                    p = np.exp(s - s.max())
                out[i, j, m] = p @ v / p.sum()
                size[i, j, m] = p @ np.abs(v) / p.sum()
                log[i, j, m] = math.log(p.sum()) + s.max() if np.isfinite(s).all() else np.nan
                reach[i, j, m] = (np.abs(k) @ np.abs(q[i, j, m])).max() * abs(scale)
    return out, log, size, reach
