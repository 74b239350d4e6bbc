"""Attention over whole sequences and its gradient where blocks, scores or values are out of the ordinary, against the forms and bounds of attention_ref."""
import pytest

from heads_ref import KIND
from test_gpu_attention import both, check, close, made, reference

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
