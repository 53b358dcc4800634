"""The table of turns against frequencies in 80 decimal digits, within the bound that include/adore.h states: 2^-65 turns and 2^-62 of the frequency."""
import math
from decimal import Decimal, getcontext
from fractions import Fraction

import pytest

from paper_2407_02328_amd.binding import Rotary

PI = Decimal("3.14159265358979323846264338327950288419716939937510582097494459230781640628620899862803482534211706798")


def exact_turns(R, base=10000.0, factor=1.0, original=None, low=1.0, high=32.0):
    """Turns per position of every pair, 80 digits."""
    getcontext().prec = 80
    turns = []
    for j in range(R // 2):
        f = Decimal(base) ** (Decimal(-2 * j) / Decimal(R)) / (2 * PI)
        whole = Decimal(0)
        if original is not None:
            whole = min(max((Decimal(original) * f - Decimal(low)) / (Decimal(high) - Decimal(low)), Decimal(0)), Decimal(1))
        turns.append(f * (whole + (1 - whole) / Decimal(factor)))
    return turns


@pytest.mark.parametrize("R,how", [
    (64, dict()), (128, dict(base=500000.0)), (32, dict(factor=4.0)), (128, dict(factor=8.0, original=4096.0)),
    (96, dict(base=1e6, factor=32.0, original=8192.0, high=4.0)), (16, dict(base=0.01)), (64, dict(base=1e-9)), (128, dict(factor=1e-6)),
    (128, dict(base=3.7, factor=0.3)), (128, dict(base=1e300))])
def test_turns_are_within_what_is_stated(R, how):
    for got, want in zip((int(t) % (1 << 64) for t in Rotary(R, **how).turns), exact_turns(R, **how)):
        off = (Fraction(got) / 2 ** 64 - Fraction(want)) % 1
        assert min(off, 1 - off) <= Fraction(1, 2 ** 65) + Fraction(want) / 2 ** 62


def test_frequencies_of_a_radian_at_most_are_within_two_roundings_at_any_position():
    """What the bound comes to for base >= 1 and factor >= 1: 2^-33 (the angle's rounding to 2^-32 turns) + 2^31 (2^-65 + 2^-62 / 2 pi)."""
    assert 2.0 ** -33 + 2.0 ** 31 * (2.0 ** -65 + 2.0 ** -62 / (2 * math.pi)) < 3 * 2.0 ** -33
