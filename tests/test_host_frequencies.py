"""Frequencies for long contexts against their definition in ocn.h, where contexts are short or long against the base (no GPU)."""
import math

import pytest

import paper_1810_08723_amd as ocn


def by_index(r, base, factor, original, low, high):
    """Mixed linearly in i between the indices where the number of turns is `high` (rounded down) and `low` (rounded up)"""
    at = lambda turns: r * math.log(original / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
    first, last = math.floor(at(high)), math.ceil(at(low))
    out = []
    for i in range(r // 2):
        share = min(1.0, max(0.0, (i - first) / (last - first)))
        f = base ** (-2 * i / r)
        out.append(f * (1 - share) + f / factor * share)
    return out, first, last


@pytest.mark.parametrize("r,base,factor,original,low,high", [
    (128, 10000.0, 4.0, 65536.0, 1.0, 32.0),      # no frequency makes as few as `low` turns: last = 65
    (64, 10000.0, 8.0, 1e6, 1.0, 4.0),
    (128, 10000.0, 4.0, 100.0, 1.0, 32.0),        # none makes as many as `high`: first < 0
    (32, 500000.0, 2.0, 10.0, 0.5, 64.0),
    (128, 10000.0, 16.0, 2.0, 1.0, 32.0),         # all make fewer than `low`: divided by factor, all of them
    (128, 10000.0, 4.0, 1e9, 1.0, 32.0),          # all make more than `high`: as they are
    (128, 10000.0, 4.0, 4096.0, 1.0, 32.0), (2, 10000.0, 4.0, 4096.0, 1.0, 32.0), (96, 1e6, 40.0, 32768.0, 1.0, 1.0625),
])
def test_index(r, base, factor, original, low, high):
    got, magnitude = ocn.rotary_frequencies(r, base, "index", factor, original, low, high)
    want, first, last = by_index(r, base, factor, original, low, high)
    assert got == pytest.approx(want, rel=1e-12) and magnitude == pytest.approx(0.1 * math.log(factor) + 1, rel=1e-14)
    if original == 2.0:
        assert last <= 0 and got == pytest.approx([base ** (-2 * i / r) / factor for i in range(r // 2)], rel=1e-12)
    if original == 1e9:
        assert first >= r // 2 and got == pytest.approx([base ** (-2 * i / r) for i in range(r // 2)], rel=1e-12)


def test_index_at_the_ends_of_the_range():
    """Parameters whose ratio leaves the range of doubles still have a logarithm"""
    got, _ = ocn.rotary_frequencies(8, 10000.0, "index", 2.0, 1e-300, 1.0, 1e300)
    assert all(math.isfinite(f) for f in got)
    got, _ = ocn.rotary_frequencies(8, 10000.0, "index", 2.0, 1e300, 1e-300, 1.0)
    assert got == pytest.approx([1.0, 0.1, 0.01, 0.001], rel=1e-12)
