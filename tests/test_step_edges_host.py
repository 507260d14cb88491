"""A decoding step's operators at the edges of what their documentation allows (no GPU)."""
import math

import pytest

import paper_2607_18957_gb300 as cfa


@pytest.mark.parametrize("dim,base,length,factor", [
    (128, 10000.0, 131072, 4.0), (128, 10000.0, 131072, 8.0), (128, 10000.0, 65536, 8.0),
    (64, 10000.0, 65536, 4.0), (64, 10000.0, 131072, 4.0), (64, 10000.0, 163840, 16.0),
    (128, 10000.0, 4096, 16.0), (64, 1e6, 32768, 4.0), (2, 10000.0, 131072, 2.0)])
def test_ramp_goes_on_behind_the_last_pair(dim, base, length, factor):
    """Pair by pair, with the ramp's ends found by counting turns instead of by logarithms: the index
    (of a pair or behind the last) from which on all turn fewer than 32 times, less one, and the first
    that turns no more than once."""
    def turns(i):
        return length * base ** (-2 * i / dim) / (2 * math.pi)
    first = next(i for i in range(10 * dim) if turns(i + 1) < 32)
    last = next(i for i in range(10 * dim) if turns(i) <= 1)
    f, _ = cfa.rotary_frequencies(dim, base, scaling="ramp", factor=factor, length=length)
    assert len(f) == dim // 2
    for i, v in enumerate(f):
        g = base ** (-2 * i / dim)
        share = min(max((i - first) / (last - first), 0.0), 1.0)  # of the frequency that is divided
        assert v == pytest.approx(g * (1 - share) + g / factor * share, rel=1e-12, abs=0.0), i


def test_ramp_leaves_pairs_that_turn_often_alone():
    """128 values, base 10000, 131,072 positions: 32 turns at index 45.03, one at 69.1, so that the last
    pair, 63, keeps 7 / 25 of its frequency and an eighth of the rest."""
    f, _ = cfa.rotary_frequencies(128, 10000.0, scaling="ramp", factor=8.0, length=131072)
    assert f[45] == pytest.approx(10000.0 ** (-45 / 64), rel=1e-12, abs=0.0)
    assert f[63] == pytest.approx(10000.0 ** (-63 / 64) * (7 / 25 + 18 / 25 / 8), rel=1e-12, abs=0.0)
