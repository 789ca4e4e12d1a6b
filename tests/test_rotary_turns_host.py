"""Frequencies' fractions of a turn for any finite number.  Nothing here reaches a device."""
import fractions
import math

import pytest


@pytest.mark.parametrize("f", [1e-300, 3.5, 1e22, 1e30, -7e31, 1e48, 1e100, 1e300, 2.0 ** 1023, -1.7e308])
def test_turns_of_any_number(f):
    """The C library's sine and cosine reduce their argument exactly: those of the fraction are the same.  Bound: 2^-65 turns, a
    double's rounding of an angle under 2 pi (2^-51) and of the functions (2^-53 each)."""
    import paper_2608_23805_amd as msi
    got = msi.KvRotary([f] * 8, device="cpu").freq
    t = 2 * math.pi * float(fractions.Fraction(int(got[0]), 2 ** 64))
    assert abs(math.sin(t) - math.sin(f)) <= 2.0 ** -50 and abs(math.cos(t) - math.cos(f)) <= 2.0 ** -50
