"""What the operators over heads refuse, before anything is launched, and a rotation's frequencies (no GPU)."""
import ctypes as C
import math

import pytest

import paper_1810_08723_amd as ocn
from paper_1810_08723_amd import binding as B

E = B.ERR
BASE = [0x1000000000 * (i + 1) for i in range(16)]


def T(dtype, sizes, strides=None, base=0, offset=0, device=0, byteswapped=False):
    size = ocn.dtype_size(dtype)
    if strides is None:
        strides, acc = [], size
        for s in reversed(sizes):
            strides.insert(0, acc)
            acc *= max(s, 1)
    return ocn.Tensor(BASE[base] if base < 16 else base, dtype, tuple(sizes), tuple(strides), offset, device, None, byteswapped)


E_NAME = {v: k for k, v in E.items()}


class FakeSpace:
    def __init__(self, at, size):
        self.at, self.size = at, size

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.size


def code(fn, *args, **kw):
    if fn is not ocn.rotary_frequencies:
        kw["stream"] = 0
    if fn in (ocn.norm_rotary_grad, ocn.cache_attention):
        kw.setdefault("workspace", FakeSpace(0x7000000000, 1 << 30))
    with pytest.raises(ocn.OcnError) as e:
        fn(*args, **kw)
    return E_NAME[e.value.code]


def rot(r=64, layout="half", pos=None, freq=None):
    return ocn.Rotation(pos or T("int32", (5,), base=8), freq or T("double", (r // 2,), base=9), r, layout)


def x(dtype="half", sizes=(5, 4, 64), **kw):
    return T(dtype, sizes, **kw)


def test_rotary_refuses():
    a, o = x(), x(base=1)
    assert code(ocn.rotary, x("double"), rot(), x("double", base=1)) == "DTYPE"
    assert code(ocn.rotary, x("int16"), rot(), x("int16", base=1)) == "DTYPE"
    assert code(ocn.rotary, a, rot(), x("bfloat16", base=1)) == "DTYPE"
    assert code(ocn.rotary, a, rot(), x(sizes=(5, 4, 32), base=1)) == "SHAPE"
    assert code(ocn.rotary, T("half", (64,)), rot(), T("half", (64,), base=1)) == "NDIM"
    assert code(ocn.rotary, a, rot(66), o) == "SHAPE"
    assert code(ocn.rotary, a, rot(63), o) == "SHAPE"
    assert code(ocn.rotary, a, ocn.Rotation(T("int32", (5,), base=8), T("double", (32,), base=9), 0), o) == "SHAPE"
    assert code(ocn.rotary, a, rot(pos=T("int32", (4,), base=8)), o) == "SHAPE"
    assert code(ocn.rotary, a, rot(pos=T("int32", (2, 5), base=8)), o) == "SHAPE"
    assert code(ocn.rotary, a, rot(pos=T("float", (5,), base=8)), o) == "DTYPE"
    assert code(ocn.rotary, a, rot(freq=T("float", (32,), base=9)), o) == "DTYPE"
    assert code(ocn.rotary, a, rot(freq=T("double", (31,), base=9)), o) == "SHAPE"
    assert code(ocn.rotary, a, rot(pos=T("int32", (5,), base=8, device=1)), o) == "DEVICE"
    assert code(ocn.rotary, a, rot(), x(base=1, device=1)) == "DEVICE"
    assert code(ocn.rotary, a, rot(), x(base=1, byteswapped=True)) == "BYTEORDER"
    assert code(ocn.rotary, a, rot(), x(base=1, offset=1)) == "ALIGN"
    assert code(ocn.rotary, x(base=0x10), rot(), T("half", (5, 4, 64), (0, 128, 2), base=1)) == "OVERLAP_OUT"
    assert code(ocn.rotary, x(offset=128), rot(), x()) == "ALIAS"
    assert code(ocn.rotary, x(sizes=(5, 4, 514)), rot(), x(sizes=(5, 4, 514), base=1)) == "SHAPE"
    lib = B.lib()
    d = a.desc()
    assert lib.ocn_rotary(C.byref(d), None, C.byref(d), 0, None) == E["NULLPTR"]
    assert lib.ocn_rotary(None, rot()._ref, C.byref(d), 0, None) == E["NULLPTR"]
    assert lib.ocn_rotary(C.byref(d), rot()._ref, C.byref(o.desc()), 4, None) == E["OP"]
    bad = rot()
    bad._struct.layout = 2
    assert code(ocn.rotary, a, bad, o) == "OP"
    with pytest.raises(AttributeError):
        bad.rotary_dim = 32
    huge = T("half", (1 << 20, 1 << 12, 1, 64), (0, 0, 128, 2))
    assert code(ocn.rotary, huge, rot(pos=T("int32", (1,), base=8)), T("half", (1 << 20, 1 << 12, 1, 64), base=0x400000000000)) == "SHAPE"


def test_bfloat16_is_a_type_of_these_operators_alone():
    a, o = T("bfloat16", (4, 8)), T("bfloat16", (4, 8), base=1)
    assert ocn.dtype_size("bfloat16") == 2
    assert code(ocn.unary, "neg", a, o) == "DTYPE" and code(ocn.binary, "add", a, a, o) == "DTYPE"
    assert code(ocn.cast_copy, a, T("float", (4, 8), base=1)) == "DTYPE" and code(ocn.reduce, "sum", a, [0], T("float", (8,), base=1)) == "DTYPE"


def test_norm_refuses():
    q, o, k, ko, w = x(), x(base=1), x(sizes=(5, 2, 64), base=2), x(sizes=(5, 2, 64), base=3), T("float", (64,), base=4)
    assert code(ocn.norm_rotary, q, T("float", (63,), base=4), o) == "SHAPE"
    assert code(ocn.norm_rotary, q, T("double", (64,), base=4), o) == "DTYPE"
    assert code(ocn.norm_rotary, q, w, o, k, None, None) == "NULLPTR"
    assert code(ocn.norm_rotary, q, w, o, x(sizes=(6, 2, 64), base=2), w, x(sizes=(6, 2, 64), base=3)) == "SHAPE"
    assert code(ocn.norm_rotary, q, w, o, x("float", sizes=(5, 2, 64), base=2), w, x("float", sizes=(5, 2, 64), base=3)) == "DTYPE"
    assert code(ocn.norm_rotary, q, w, o, k, w, o) == "SHAPE"
    assert code(ocn.norm_rotary, q, w, o, x(base=2), w, o) == "ALIAS"             # two outputs in one place
    assert code(ocn.norm_rotary, q, T("half", (64,), base=1), o) == "ALIAS"
    # queries and keys side by side share nothing, and may be normed in place; overlapping heads share
    row = (12 * 128, 128, 2)
    a, b = T("half", (5, 8, 64), row), T("half", (5, 2, 64), row, offset=8 * 128)
    lib = B.lib()
    assert code(ocn.norm_rotary, a, w, a, T("half", (5, 2, 64), row, offset=7 * 128), w, ko) == "ALIAS"
    assert code(ocn.norm_rotary, a, w, a, b, T("float", (64,), base=4, device=1), b) == "DEVICE"      # (got past the sharing)
    g, gi, gw = x(base=5), x(base=6), T("float", (64,), base=7)
    assert code(ocn.norm_rotary_grad, g, q, None, gi, gw, workspace=FakeSpace(0x7000000000, 1 << 20)) == "NULLPTR"
    assert code(ocn.norm_rotary_grad, g, q, w, gi, T("float", (1,), base=7)) == "SHAPE"
    assert code(ocn.norm_rotary_grad, x("float", base=5), q, w, gi, gw) == "DTYPE"
    assert code(ocn.norm_rotary_grad, g, q, w, x(base=5, offset=128), gw) == "ALIAS"
    need = ocn.norm_rotary_grad_workspace_bytes(q)
    assert need > 0 and need % (64 * 4) == 0
    assert code(ocn.norm_rotary_grad, g, q, w, gi, gw, workspace=FakeSpace(0x7000000000, need - 1)) == "WORKSPACE"
    assert code(ocn.norm_rotary_grad, g, q, w, gi, gw, workspace=FakeSpace(0x7000000010, need)) == "ALIGN"
    assert lib.ocn_norm_rotary_grad_workspace_bytes(None, None) == 0
    assert ocn.norm_rotary_grad_workspace_bytes(x("double")) == 0


def cache_of(pages=7, heads=4, page=16, d=64, **kw):
    return T("uint8", (pages, heads, ocn.cache_block_bytes(page, d)), **kw)


def test_block_bytes():
    assert ocn.cache_block_bytes(16, 128) == 2304 and ocn.cache_block_bytes(48, 64) == 3456 and ocn.cache_block_bytes(128, 256) == 36864
    assert [ocn.cache_block_bytes(p, d) for p, d in ((0, 64), (8, 64), (17, 64), (16, 96), (16, 512), (-16, 64), (1 << 40, 64))] == [0] * 7


def test_append_and_read_refuse():
    k, v, s = x(), x(base=1), T("int64", (5,), base=2)
    c = cache_of(base=3)
    assert code(ocn.cache_append, k, x(sizes=(5, 3, 64), base=1), s, c) == "SHAPE"
    assert code(ocn.cache_append, k, x("float", base=1), s, c) == "DTYPE"
    assert code(ocn.cache_append, k, v, T("int64", (4,), base=2), c) == "SHAPE"
    assert code(ocn.cache_append, k, v, T("int64", (1, 5), base=2), c) == "SHAPE"
    assert code(ocn.cache_append, k, v, T("half", (5,), base=2), c) == "DTYPE"
    assert code(ocn.cache_append, k, v, s, cache_of(heads=3, base=3)) == "SHAPE"
    assert code(ocn.cache_append, k, v, s, T("uint8", (7, 4, 1150), base=3)) == "SHAPE"
    assert code(ocn.cache_append, k, v, s, T("int8", (7, 4, 1152), base=3)) == "DTYPE"
    assert code(ocn.cache_append, k, v, s, T("uint8", (7, 4, 1152), (4 * 1152 + 8, 1152, 1), base=3)) == "ALIGN"
    assert code(ocn.cache_append, k, v, s, cache_of(base=3, offset=8)) == "ALIGN"
    assert code(ocn.cache_append, k, v, s, T("uint8", (7, 4, 1152), (1152, 0, 1), base=3)) == "OVERLAP_OUT"
    assert code(ocn.cache_append, x(sizes=(5, 4, 96)), x(sizes=(5, 4, 96), base=1), s, c) == "SHAPE"
    assert code(ocn.cache_append, k, x(base=3), s, c) == "ALIAS"
    assert code(ocn.cache_append, k, v, s, c, rotation=rot(128)) == "SHAPE"
    assert code(ocn.cache_read, c, s, None, None) == "NULLPTR"
    assert code(ocn.cache_read, c, s, k, x("float", base=1)) == "DTYPE"
    assert code(ocn.cache_read, c, s, k, k) == "ALIAS"
    assert code(ocn.cache_read, c, s, T("half", (5, 4, 64), (512, 0, 2)), None) == "OVERLAP_OUT"
    lib = B.lib()
    assert lib.ocn_cache_append(None, C.byref(v.desc()), None, C.byref(s.desc()), C.byref(c.desc()), None) == E["NULLPTR"]
    assert lib.ocn_cache_append(C.byref(k.desc()), C.byref(v.desc()), None, None, C.byref(c.desc()), None) == E["NULLPTR"]


def test_attention_refuses():
    q, o = T("half", (2, 3, 8, 64)), T("half", (2, 3, 8, 64), base=1)
    c, t, n = cache_of(base=3), T("int32", (2, 9), base=4), T("int64", (2, 3), base=5)
    f = ocn.cache_attention
    assert code(f, T("half", (3, 8, 64)), c, t, n, o, 0.1) == "NDIM"
    assert code(f, T("double", (2, 3, 8, 64)), c, t, n, o, 0.1) == "DTYPE"
    assert code(f, T("half", (2, 3, 6, 64)), c, t, n, T("half", (2, 3, 6, 64), base=1), 0.1) == "SHAPE"
    assert code(f, T("half", (2, 3, 8, 96)), c, t, n, T("half", (2, 3, 8, 96), base=1), 0.1) == "SHAPE"
    assert code(f, q, c, T("int32", (3, 9), base=4), n, o, 0.1) == "SHAPE"
    assert code(f, q, c, T("int32", (2,), base=4), n, o, 0.1) == "NDIM"
    assert code(f, q, c, T("uint8", (2, 9), base=4), n, o, 0.1) == "DTYPE"
    assert code(f, q, c, t, T("int32", (2, 2), base=5), o, 0.1) == "SHAPE"
    assert code(f, q, c, t, T("int32", (2,), base=5), o, 0.1) == "NDIM"
    assert code(f, q, c, t, n, T("bfloat16", (2, 3, 8, 64), base=1), 0.1) == "DTYPE"
    assert code(f, q, c, t, n, T("half", (2, 4, 8, 64), base=1), 0.1) == "SHAPE"
    assert code(f, q, c, t, n, o, math.inf) == "DOMAIN"
    assert code(f, q, c, t, n, o, math.nan) == "DOMAIN"
    assert code(f, q, c, t, n, o, 0.1, window=-1) == "DOMAIN"
    assert code(f, q, c, t, n, o, 0.1, log_sum=T("half", (2, 3, 8), base=6)) == "DTYPE"
    assert code(f, q, c, t, n, o, 0.1, log_sum=T("float", (2, 3, 4), base=6)) == "SHAPE"
    assert code(f, q, c, t, n, T("half", (2, 3, 8, 64), base=0, offset=128), 0.1) == "ALIAS"
    assert code(f, q, c, T("int32", (2, 9), base=1), n, o, 0.1) == "ALIAS"
    assert code(f, q, c, T("int32", (2, 1 << 28), base=4), n, o, 0.1) == "SHAPE"
    assert code(f, q, c, T("int32", (2, 9), base=4, device=1), n, o, 0.1) == "DEVICE"


def test_frequencies():
    f, m = ocn.rotary_frequencies(8)
    assert m == 1.0 and f == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-15)
    f, m = ocn.rotary_frequencies(8, stretch="linear", factor=4.0)
    assert m == 1.0 and f == pytest.approx([0.25, 0.025, 0.0025, 0.00025], rel=1e-15)
    f, m = ocn.rotary_frequencies(8, stretch="base", factor=16.0)
    assert f == pytest.approx([(10000 * 16 ** (8 / 6)) ** (-i / 4) for i in range(4)], rel=1e-14)
    assert f[3] == pytest.approx(0.001 / 16, rel=1e-13)                     # the slowest is divided by factor
    # turns within 1000 tokens: 159.2, 15.92, 1.592, 0.1592
    f, m = ocn.rotary_frequencies(8, stretch="turns", factor=10.0, original=1000.0, low=1.0, high=4.0)
    share = (1000 * 0.01 / (2 * math.pi) - 1) / 3
    assert m == 1.0 and f == pytest.approx([1.0, 0.1, 0.01 * share + 0.001 * (1 - share), 0.0001], rel=1e-14)
    # indices where a frequency makes 32 and 1 turns within 4096 tokens
    f, m = ocn.rotary_frequencies(128, stretch="index", factor=4.0, original=4096.0, low=1.0, high=32.0)
    at = lambda turns: 128 * math.log(4096 / (turns * 2 * math.pi)) / (2 * math.log(10000.0))  # noqa: E731
    first, last = math.floor(at(32)), math.ceil(at(1))
    for i, got in enumerate(f):
        ramp = min(1.0, max(0.0, (i - first) / (last - first)))
        plain = 10000.0 ** (-i / 64)
        assert got == pytest.approx(plain * (1 - ramp) + plain / 4 * ramp, rel=1e-13)
    assert m == pytest.approx(0.1 * math.log(4) + 1)
    for kw in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, base=1.0), dict(rotary_dim=8, base=math.inf), dict(rotary_dim=8, stretch="linear", factor=0.0),
               dict(rotary_dim=2, stretch="base", factor=2.0), dict(rotary_dim=8, stretch="turns", factor=2.0, original=0.0),
               dict(rotary_dim=8, stretch="index", factor=2.0, original=100.0, low=4.0, high=4.0)):
        assert code(ocn.rotary_frequencies, **kw) == "SHAPE"


def test_attention_refuses_scales_past_single_precision():
    q, o = T("half", (2, 3, 8, 64)), T("half", (2, 3, 8, 64), base=1)
    c, t, n = cache_of(base=3), T("int32", (2, 9), base=4), T("int64", (2, 3), base=5)
    for scale in (3e38, -3e38, 1e300):
        assert code(ocn.cache_attention, q, c, t, n, o, scale) == "DOMAIN"
