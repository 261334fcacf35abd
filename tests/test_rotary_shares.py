"""Frequencies as shares of a turn: integers of 64 bits, the nearest ones to the doubles that Rotary.frequencies gives."""
import math
from fractions import Fraction

import pytest

# pi to 100 digits
PI = Fraction(31415926535897932384626433832795028841971693993751058209749445923078164062862089986280348253421170679, 10 ** 100)


@pytest.fixture(scope="module")
def P():
    pytest.importorskip("torch")
    import paper_2608_19677_gb300 as P
    return P


def off_by(turn, f):
    """Units of 2^-64 turns between an integer and the frequency f, whole turns left out."""
    d = (turn - Fraction(f) / (2 * PI) * 2 ** 64) % 2 ** 64
    return float(min(d, 2 ** 64 - d))


@pytest.mark.parametrize("how", [dict(), dict(base=500000.0), dict(scaling="linear", factor=8.0), dict(scaling="ntk", factor=4.0),
                                 dict(scaling="ramp", factor=16.0, original=4096),
                                 dict(frequencies=[6.5, -0.25, 2 * math.pi, 1e-9, -1e-30, 0.0, 123456.789, 2.0 ** 40] + [1.0 / (i + 3) for i in range(56)])])
def test_shares_are_the_nearest_integers(P, how):
    """Half a unit at most: pi's digits leave 1e-70 of it."""
    r = P.Rotary(128, device="cpu", **how)
    for t, f in zip(r.turn.tolist(), r.frequencies):
        assert off_by(t, f) <= 0.5 * (1 + 1e-12), f


def test_frequencies_that_are_no_numbers_are_refused(P):
    for wrong in (dict(scaling="linear", factor=1e-320), dict(base=1e-320), dict(scaling="ntk", factor=1e300, base=1e300)):
        with pytest.raises(ValueError):
            P.Rotary(128, device="cpu", **wrong)
