"""Frequencies in parts where contexts are short, bases small and turn counts large, so that
the ramp between the two turn counts lies partly or wholly outside the pairs (CPU)."""
import math

import numpy as np
import pytest

jfkv = pytest.importorskip("paper_2609_17475_amd.jfkv")


@pytest.mark.parametrize("rot", [2, 4, 6, 64, 128])
@pytest.mark.parametrize("base", [1.5, 10.0, 10000.0, 500000.0])
def test_pairs_by_their_turns(rot, base):
    """The definition: pairs of more than `fast` turns in original_len positions stay, those
    of fewer than `slow` are divided, those between lie between."""
    f = float(base) ** (-2 * np.arange(rot // 2, dtype=np.longdouble) / rot)
    sides = np.zeros(3, int)
    for length in (1, 2, 3, 6, 7, 30, 200, 201, 202, 4096, 10 ** 6, 2 ** 31 - 1):
        for fast, slow in ((32.0, 1.0), (2.0, 1.0), (64.0, 32.0), (1e4, 1e3), (1e-3, 1e-4)):
            got = jfkv.rope_frequencies(rot, base, "parts", 4.0, length, fast, slow)[0].numpy().astype(np.longdouble)
            turns = length * f / (2 * math.pi)
            # (a pair at a border, within the roundings of 64 bits, may count to either side)
            few, many = turns < slow * (1 - 1e-9), turns > fast * (1 + 1e-9)
            tol = f * (2.0 ** -24 + 2.0 ** -40)  # one rounding to fp32, some in 64 bits
            assert np.all(np.abs(got - f / 4)[few] <= tol[few]), (length, fast, slow)
            assert np.all(np.abs(got - f)[many] <= tol[many]), (length, fast, slow)
            assert np.all(got >= f / 4 - tol) and np.all(got <= f + tol)
            sides += few.sum(), many.sum(), (~few & ~many).sum()
    assert sides[0] and sides[1]


def test_the_first_pair_of_a_short_context():
    # 6 positions are 0.95 of a turn of the first pair, 200 are 31.8
    for rot, length, fast, slow in ((64, 6, 32.0, 1.0), (64, 1, 2.0, 1.0), (2, 3, 32.0, 1.0), (128, 200, 64.0, 32.0)):
        got = jfkv.rope_frequencies(rot, 10000.0, "parts", 8.0, length, fast, slow)[0]
        assert got[0] == 0.125, (rot, length)
    # and of a context in which every pair turns often enough
    got = jfkv.rope_frequencies(4, 1.5, "parts", 8.0, 10 ** 6, 32.0, 1.0)[0]
    assert got[0] == 1.0 and abs(float(got[1]) - 1.5 ** -0.5) < 1e-7
