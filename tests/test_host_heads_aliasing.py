"""Which operands of the operators over heads may share bytes: told by their place in a call, not by the descriptor that names them (no GPU)."""
import paper_1810_08723_amd as ocn
from test_host_heads import FakeSpace, T, code, rot, x

W = T("float", (64,), base=4)


def test_one_descriptor_for_queries_and_keys():
    """Written in place of the queries, the keys' heads would be read while they change"""
    q, out = x(), x(base=3)
    for weight in (W, None):
        assert code(ocn.norm_rotary, q, weight, q, q, weight, out) == "ALIAS"
        assert code(ocn.norm_rotary, q, weight, out, q, weight, q) == "ALIAS"
        assert code(ocn.norm_rotary, q, weight, q, q, weight, q) == "ALIAS"
    g, gin = x(base=5), x(base=6)
    f = ocn.norm_rotary_grad
    assert code(f, g, q, W, q, None, x(base=7), q, W, gin) == "ALIAS"            # the keys are read for their own gradient
    assert code(f, g, q, W, g, None, g, x(base=7), W, gin) == "ALIAS"            # one gradient of both outputs
    assert code(f, g, q, W, gin, None, g, x(base=7), W, g) == "ALIAS"


def test_what_may_be_in_place_still_is():
    """Such calls are refused later: for positions that fit no call, or for too small a workspace"""
    q, k, g, kg = x(), x(base=3), x(base=5), x(base=6)
    off = rot(2, pos=T("int32", (1000,), base=8))
    assert code(ocn.norm_rotary, q, W, q, k, W, k, rotation=off) == "SHAPE"
    assert code(ocn.norm_rotary, q, W, x(base=7), q, W, k, rotation=off) == "SHAPE"        # read twice, written elsewhere
    f, gw, small = ocn.norm_rotary_grad, T("float", (64,), base=9), FakeSpace(0x7000000000, 16)
    assert code(f, g, q, W, g, gw, kg, k, W, k, workspace=small) == "WORKSPACE"
    assert code(f, q, q, W, q, gw, kg, k, W, kg, workspace=small) == "WORKSPACE"           # (the gradient of half the sum of squares)
