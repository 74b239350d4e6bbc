"""What attention over whole sequences, the layer norm and rotations with several axes refuse, before anything is launched (no GPU)."""
import ctypes as C
import math

import pytest

import paper_1810_08723_amd as ocn
from paper_1810_08723_amd import binding as B
from test_host_heads import BASE, E, FakeSpace, T, code

ROOM = 0x700000000000


def space(size=1 << 40, at=ROOM):
    return FakeSpace(at, size)


def packed(dtype="half", tokens=9, heads=8, channels=64, base=0, **kw):
    return T(dtype, (tokens, heads, channels), base=base, **kw)


def starts(n=3, base=8, dtype="int32", **kw):
    return T(dtype, (n,), base=base, **kw)


class Attention:
    """arguments that are taken, each of which a test replaces"""

    def __init__(self):
        self.a = dict(q=packed(), k=packed(tokens=12, heads=2, base=1), v=packed(tokens=12, heads=2, base=2), out=packed(base=3), scale=0.1, q_starts=starts(),
                      k_starts=starts(base=9), workspace=space())
        self.g = dict(self.a, gout=packed(base=4), log_sum=T("float", (9, 8), base=5), q_gin=packed(base=6), k_gin=packed(tokens=12, heads=2, base=7),
                      v_gin=packed(tokens=12, heads=2, base=10))

    def refused(self, **kw):
        return code(ocn.attention, **dict(self.a, **kw))

    def grad_refused(self, **kw):
        return code(ocn.attention_grad, **dict(self.g, **kw))

    def both(self, **kw):
        a, b = self.refused(**kw), self.grad_refused(**kw)
        assert a == b
        return a


# every argument of both calls
@pytest.mark.parametrize("change,error", [
    (dict(q=packed("double")), "DTYPE"), (dict(k=packed("bfloat16", tokens=12, heads=2, base=1)), "DTYPE"), (dict(v=packed("float", tokens=12, heads=2, base=2)), "DTYPE"),
    (dict(out=packed("float", base=3)), "DTYPE"), (dict(q_starts=starts(dtype="uint8")), "DTYPE"), (dict(k_starts=starts(base=9, dtype="float")), "DTYPE"),
    (dict(q=T("half", (9, 64))), "NDIM"), (dict(q=T("half", (1, 9, 8, 64))), "NDIM"), (dict(k=T("half", (12, 64), base=1)), "NDIM"), (dict(q_starts=T("int32", (1, 3), base=8)), "NDIM"),
    (dict(k_starts=T("int32", (), base=9)), "NDIM"), (dict(q=packed(heads=7), out=packed(heads=7, base=3)), "SHAPE"), (dict(q=packed(channels=60), out=packed(channels=60, base=3)), "SHAPE"),
    (dict(k=packed(tokens=12, heads=0, base=1), v=packed(tokens=12, heads=0, base=2)), "SHAPE"), (dict(v=packed(tokens=11, heads=2, base=2)), "SHAPE"),
    (dict(v=packed(tokens=12, heads=2, channels=32, base=2)), "SHAPE"), (dict(out=packed(tokens=8, base=3)), "SHAPE"), (dict(q_starts=starts(4)), "SHAPE"), (dict(k_starts=starts(0, base=9)), "SHAPE"),
    (dict(q_starts=starts(0), k_starts=starts(0, base=9)), "SHAPE"),
    (dict(q_starts=None), "NULLPTR"), (dict(k_starts=None), "NULLPTR"), (dict(q_starts=None, k_starts=None), "NDIM"),
    (dict(q=None), "NULLPTR"), (dict(k=None), "NULLPTR"), (dict(v=None), "NULLPTR"), (dict(out=None), "NULLPTR"), (dict(q=ocn.Tensor(0, "half", (9, 8, 64), (1024, 128, 2))), "NULLPTR"),
    (dict(window=-1), "SHAPE"), (dict(window=5, causal=False), "SHAPE"), (dict(window=-5, causal=False), "SHAPE"),
    (dict(scale=math.inf), "DOMAIN"), (dict(scale=math.nan), "DOMAIN"), (dict(scale=-3e38), "DOMAIN"),
    (dict(q=packed(byteswapped=True)), "BYTEORDER"), (dict(k_starts=starts(base=9, byteswapped=True)), "BYTEORDER"),
    (dict(q=packed(offset=1)), "ALIGN"), (dict(k=T("half", (12, 2, 64), (257, 128, 2), base=1)), "ALIGN"), (dict(q_starts=starts(offset=2)), "ALIGN"),
    (dict(v=packed(tokens=12, heads=2, base=2, device=1)), "DEVICE"), (dict(k_starts=starts(base=9, device=1)), "DEVICE"),
    (dict(workspace=space(at=ROOM + 16)), "ALIGN"),
], ids=lambda c: "-".join(c) if isinstance(c, dict) else c)
def test_both_refuse(change, error):
    a = Attention()
    if "workspace" in change:            # (few rows over long keys need one)
        a.a.update(k=packed(tokens=5000, heads=2, base=1), v=packed(tokens=5000, heads=2, base=2))
        a.g.update(a.a, k_gin=packed(tokens=5000, heads=2, base=7), v_gin=packed(tokens=5000, heads=2, base=10))
    assert a.both(**change) == error


def test_channels_and_sizes_past_the_limits():
    a = Attention()
    wide = {n: T("half", t.sizes[:2] + (257,), base=i) for i, (n, t) in enumerate((n, a.g[n]) for n in ("q", "k", "v", "out", "gout", "q_gin", "k_gin", "v_gin"))}
    assert a.refused(**{n: wide[n] for n in ("q", "k", "v", "out")}) == "SHAPE" and a.grad_refused(**wide) == "SHAPE"
    # 2^31 rows over all heads, and 2^31 keys
    many = dict(q=T("half", (1 << 28, 8, 64), (0, 128, 2)), out=T("half", (1 << 28, 8, 64), base=3))
    assert a.refused(**many) == "SHAPE"
    keys = dict(k=T("half", (1 << 31, 2, 64), (0, 128, 2), base=1), v=T("half", (1 << 31, 2, 64), (0, 128, 2), base=2))
    assert a.refused(**keys) == "SHAPE"
    for tokens, error in (((1 << 30) + 1, "SHAPE"), (1 << 30, "DEVICE")):      # (sums of positions are held in 32 bits; the second gets past the sizes)
        keys = dict(k=T("half", (tokens, 2, 64), (0, 128, 2), base=1), v=T("half", (tokens, 2, 64), (0, 128, 2), base=2, device=1))
        assert a.refused(**keys) == error
        queries = dict(q=T("half", (tokens, 1, 64), (0, 128, 2)), k=packed(tokens=12, heads=1, base=1), v=packed(tokens=12, heads=1, base=2), out=T("half", (tokens, 1, 64), base=3, device=1))
        assert a.refused(**queries) == error
    batch = dict(q_starts=None, k_starts=None, q=T("half", (1 << 16, 1 << 15, 2, 64), (0, 0, 128, 2)), k=T("half", (1 << 16, 4, 2, 64), (0, 0, 128, 2), base=1),
                 v=T("half", (1 << 16, 4, 2, 64), (0, 0, 128, 2), base=2), out=T("half", (1 << 16, 1 << 15, 2, 64), base=3))
    assert a.refused(**batch) == "SHAPE"
    assert a.refused(q_starts=None, k_starts=None, q=T("half", (2, 9, 8, 64)), k=T("half", (3, 9, 8, 64), base=1), v=T("half", (3, 9, 8, 64), base=2),
                     out=T("half", (2, 9, 8, 64), base=3)) == "SHAPE"
    for t in (a.a["q"], T("double", (9, 8, 64)), T("half", (9, 8, 257))):
        lib = B.lib()
        assert (lib.ocn_attention_grad_workspace_bytes(C.byref(t.desc()), C.byref(a.a["k"].desc()), C.byref(starts().desc())) > 0) == (t is a.a["q"])
    assert lib.ocn_attention_workspace_bytes(None, None, None) == 0 and lib.ocn_attention_grad_workspace_bytes(None, None, None) == 0


def test_attention_refuses_outputs():
    a = Attention()
    assert a.refused(out=packed(base=0)) == "ALIAS" and a.refused(out=packed(base=0, offset=256)) == "ALIAS"
    assert a.refused(out=T("half", (9, 8, 64), base=BASE[1] - 64)) == "ALIAS" and a.refused(out=packed(base=2)) == "ALIAS"
    assert a.refused(q_starts=starts(base=3)) == "ALIAS"
    assert a.refused(out=T("half", (9, 8, 64), (0, 128, 2), base=3)) == "OVERLAP_OUT"
    sums = lambda dtype="float", sizes=(9, 8), **kw: T(dtype, sizes, **dict(dict(base=5), **kw))  # noqa: E731
    assert a.refused(log_sum=sums("half")) == "DTYPE" and a.refused(log_sum=sums("double")) == "DTYPE"
    assert a.refused(log_sum=sums(sizes=(9, 4))) == "SHAPE" and a.refused(log_sum=sums(sizes=(9,))) == "NDIM"
    assert a.refused(log_sum=sums(strides=(0, 4))) == "OVERLAP_OUT" and a.refused(log_sum=sums(base=3)) == "ALIAS"
    assert a.refused(log_sum=sums(device=1)) == "DEVICE" and a.refused(log_sum=sums(byteswapped=True)) == "BYTEORDER"


def test_attention_workspace():
    a = Attention()
    long = dict(k=packed(tokens=5000, heads=2, base=1), v=packed(tokens=5000, heads=2, base=2))
    need = ocn.attention_workspace_bytes(a.a["q"], long["k"], a.a["q_starts"])
    assert need > 0
    assert a.refused(**long, workspace=space(need - 1)) == "WORKSPACE"
    need = ocn.attention_grad_workspace_bytes(a.g["q"], a.g["k"], a.g["q_starts"])
    assert need > 0 and need % 256 == 0
    assert a.grad_refused(workspace=space(need - 1)) == "WORKSPACE"
    # a function of the shapes alone
    strided = T("half", (9, 8, 64), (4096, 256, 4))
    assert ocn.attention_grad_workspace_bytes(strided, a.g["k"], starts(base=11)) == need


def test_attention_grad_refuses():
    a = Attention()
    assert a.grad_refused(log_sum=None) == "NULLPTR" and a.grad_refused(gout=None) == "NULLPTR"
    assert a.grad_refused(k_gin=None) == "NULLPTR" and a.grad_refused(v_gin=None) == "NULLPTR"
    assert a.grad_refused(gout=packed("float", base=4)) == "DTYPE" and a.grad_refused(q_gin=packed("float", base=6)) == "DTYPE"
    assert a.grad_refused(gout=packed(tokens=8, base=4)) == "SHAPE" and a.grad_refused(q_gin=packed(heads=4, base=6)) == "SHAPE"
    assert a.grad_refused(k_gin=packed(tokens=12, heads=8, base=7)) == "SHAPE" and a.grad_refused(v_gin=packed(tokens=13, heads=2, base=10)) == "SHAPE"
    assert a.grad_refused(log_sum=T("float", (8, 9), base=5)) == "SHAPE" and a.grad_refused(log_sum=T("half", (9, 8), base=5)) == "DTYPE"
    for name, base in (("q_gin", 0), ("q_gin", 4), ("k_gin", 1), ("v_gin", 2), ("q_gin", 3), ("k_gin", 5)):
        t = a.g[name]
        assert a.grad_refused(**{name: T("half", t.sizes, base=base)}) == "ALIAS", (name, base)
    assert a.grad_refused(v_gin=T("half", (12, 2, 64), base=7)) == "ALIAS"
    assert a.grad_refused(k_gin=T("half", (12, 2, 64), (256, 0, 2), base=7)) == "OVERLAP_OUT"
    assert a.grad_refused(q_gin=packed(base=6, device=2)) == "DEVICE"


def test_flags_that_there_are_not():
    a = Attention().a
    args = [C.byref(a[n].desc()) for n in ("q", "k", "v", "q_starts", "k_starts")]
    for flags in (1, 2, 8, 12, 1 << 31):
        assert B.lib().ocn_attention(*args, 0.1, 0, flags, C.byref(a["out"].desc()), None, ROOM, 1 << 40, None) == E["OP"]


def test_nothing_to_do_is_no_error():
    q, k = packed(tokens=0), packed(tokens=12, heads=2, base=1)
    assert ocn.attention(q, k, packed(tokens=12, heads=2, base=2), packed(tokens=0, base=3), 0.1, starts(), starts(base=9), stream=0, workspace=space()) is None
    assert ocn.attention(packed(), k, packed(tokens=12, heads=2, base=2), packed(base=3), 0.1, starts(1), starts(1, base=9), stream=0, workspace=space()) is None
    g = Attention().g
    assert ocn.attention_grad(**dict(g, q_gin=None, k_gin=None, v_gin=None), stream=0) is None
    x = T("float", (0, 64))
    assert ocn.layer_norm(x, None, None, T("float", (0, 64), base=1), stream=0) is None
    assert ocn.layer_norm(T("float", (4, 0)), None, None, T("float", (4, 0), base=1), stream=0) is None
    assert ocn.layer_norm_grad(x, T("float", (0, 64), base=1), None, T("float", (0, 64), base=2), stream=0) is None


def test_layer_norm_refuses():
    x, o, w, b = T("half", (5, 64)), T("half", (5, 64), base=1), T("float", (64,), base=2), T("bfloat16", (64,), base=3)
    f = ocn.layer_norm
    assert code(f, T("double", (5, 64)), w, b, T("double", (5, 64), base=1)) == "DTYPE"
    assert code(f, x, w, b, T("float", (5, 64), base=1)) == "DTYPE"
    assert code(f, x, T("double", (64,), base=2), b, o) == "DTYPE" and code(f, x, w, T("int32", (64,), base=3), o) == "DTYPE"
    assert code(f, x, T("float", (63,), base=2), b, o) == "SHAPE" and code(f, x, w, T("float", (1,), base=3), o) == "SHAPE"
    assert code(f, x, w, b, T("half", (5, 63), base=1)) == "SHAPE" and code(f, x, w, b, T("half", (4, 64), base=1)) == "SHAPE"
    assert code(f, x, T("float", (1, 64), base=2), b, o) in ("NDIM", "SHAPE")
    assert code(f, T("half", ()), None, None, T("half", (), base=1)) == "NDIM"
    assert code(f, T("half", (1,) * 7 + (64,)), None, None, T("half", (1,) * 7 + (64,), base=1)) == "NDIM"
    assert code(f, T("half", (2, 16385)), None, None, T("half", (2, 16385), base=1)) == "SHAPE"
    assert code(f, T("half", (1 << 16, 1 << 15, 4), (0, 0, 2)), None, None, T("half", (1 << 16, 1 << 15, 4), base=1)) == "SHAPE"
    assert code(f, x, w, b, T("half", (5, 64), base=1, byteswapped=True)) == "BYTEORDER"
    assert code(f, x, w, b, T("half", (5, 64), base=1, device=1)) == "DEVICE" and code(f, x, T("float", (64,), base=2, device=1), b, o) == "DEVICE"
    assert code(f, T("half", (5, 64), offset=1), w, b, o) == "ALIGN" and code(f, x, T("float", (64,), base=2, offset=2), b, o) == "ALIGN"
    assert code(f, x, w, b, T("half", (5, 64), (0, 2), base=1)) == "OVERLAP_OUT"
    assert code(f, x, w, b, T("half", (5, 64), offset=128)) == "ALIAS" and code(f, x, T("half", (64,), base=1), b, o) == "ALIAS"
    lib, d = B.lib(), C.byref(x.desc())
    assert lib.ocn_layer_norm(None, None, None, d, 1e-5, None) == E["NULLPTR"] and lib.ocn_layer_norm(d, None, None, None, 1e-5, None) == E["NULLPTR"]


def test_layer_norm_grad_refuses():
    x, g, gi, w = T("half", (5, 64)), T("half", (5, 64), base=1), T("half", (5, 64), base=2), T("float", (64,), base=3)
    gw, gb, f = T("float", (64,), base=4), T("half", (64,), base=5), ocn.layer_norm_grad
    room = dict(workspace=space())
    assert code(f, T("float", (5, 64), base=1), x, w, gi, gw, gb, **room) == "DTYPE" and code(f, g, x, w, T("float", (5, 64), base=2), gw, gb, **room) == "DTYPE"
    assert code(f, g, x, w, gi, T("double", (64,), base=4), gb, **room) == "DTYPE"
    assert code(f, T("half", (4, 64), base=1), x, w, gi, gw, gb, **room) == "SHAPE" and code(f, g, x, w, gi, gw, T("half", (65,), base=5), **room) == "SHAPE"
    assert code(f, g, x, None, gi, gw, gb, **room) == "NULLPTR"                     # a weight's gradient without a weight
    assert code(f, g, x, w, gi, T("float", (64,), (0,), base=4), gb, **room) == "OVERLAP_OUT"
    assert code(f, g, x, w, gi, T("float", (64,), base=3), gb, **room) == "ALIAS" and code(f, g, x, w, gi, gw, T("float", (64,), base=4), **room) == "ALIAS"
    assert code(f, g, x, w, T("half", (5, 64), base=1, offset=128), gw, gb, **room) == "ALIAS"
    assert code(f, g, x, w, gi, T("float", (64,), base=4, device=1), gb, **room) == "DEVICE"
    need = ocn.layer_norm_grad_workspace_bytes(x)
    assert need > 0 and need % (2 * 64 * 4) == 0
    assert code(f, g, x, w, gi, gw, None, workspace=space(need - 1)) == "WORKSPACE" and code(f, g, x, w, gi, None, gb, workspace=space(need, ROOM + 64)) == "ALIGN"
    assert ocn.layer_norm_grad_workspace_bytes(T("double", (5, 64))) == 0 and B.lib().ocn_layer_norm_grad_workspace_bytes(None) == 0
    lib, d = B.lib(), C.byref(x.desc())
    for missing in range(3):
        args = [None if i == missing else d for i in range(2)] + [None, None if missing == 2 else d, None, None, 1e-5, None, 0, None]
        assert lib.ocn_layer_norm_grad(*args) == E["NULLPTR"]


def test_several_axes():
    f = [1.0, 0.5, 0.25, 0.125, 0.0625]
    assert ocn.rotary_axes([2, 0, 3], f) == [[1.0, 0.5, 0, 0, 0], [0] * 5, [0, 0, 0.25, 0.125, 0.0625]]
    assert ocn.rotary_axes([1, 2, 2], f, "turn") == [[1.0, 0, 0, 0, 0], [0, 0.5, 0, 0.125, 0], [0, 0, 0.25, 0, 0.0625]]
    assert ocn.rotary_axes([5], f) == [f] and ocn.rotary_axes([5], f, "turn") == [f]
    assert ocn.rotary_axes([0, 0, 0, 256], [0.5] * 256)[3] == [0.5] * 256
    for pairs in ([], [-1, 6], [1] * 5, [0, 0], [0, 257]):
        with pytest.raises(ocn.OcnError) as e:
            ocn.rotary_axes(pairs, [1.0] * max(sum(pairs), 0))
        assert e.value.code == E["SHAPE"], pairs
    with pytest.raises(ValueError):
        ocn.rotary_axes([2, 2], f)
    with pytest.raises(ValueError):
        ocn.rotary_axes([2, 3], f, "column")
    lib, one = B.lib(), (C.c_int32 * 1)(1)
    room = (C.c_double * 1)(1.0)
    assert lib.ocn_rotary_axes(1, one, 2, room, room) == E["OP"]
    assert lib.ocn_rotary_axes(1, None, 0, room, room) == lib.ocn_rotary_axes(1, one, 0, None, room) == lib.ocn_rotary_axes(1, one, 0, room, None) == E["NULLPTR"]


def test_rotations_of_several_axes_refuse():
    x, o = T("half", (5, 4, 64)), T("half", (5, 4, 64), base=1)
    rot = lambda pos, freq, r=64: ocn.Rotation(T("int32", pos, base=8), T("double", freq, base=9), r, "half")  # noqa: E731
    for pos, freq in (((5,), (3, 32)), ((2, 5), (3, 32)), ((), (1, 32)), ((3, 4), (3, 32)), ((3, 2, 5), (3, 32)), ((5, 5), (5, 32)), ((3, 5), (3, 31)), ((0, 5), (0, 32)), ((3, 5), (1, 3, 32))):
        assert code(ocn.rotary, x, rot(pos, freq), o) in ("SHAPE", "NDIM"), (pos, freq)
    assert code(ocn.rotary, x, rot((3, 5), (3, 32)), T("half", (5, 4, 64), base=1, device=1)) == "DEVICE"      # (got past the sizes)
