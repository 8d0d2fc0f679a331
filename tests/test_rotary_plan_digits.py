"""The frequencies of a rotation to the last of their 64 bits, against whole-number arithmetic: logarithms, exponentials and pi from
their series with 400 bits behind the point.  No GPU is needed."""
import math
from fractions import Fraction

import pytest

import paper_2107_03474_amd as lram

BITS = 400
ONE = 1 << BITS


def _fixed(x):
    return int(Fraction(x) * ONE)


def _atanh(x):  # of a rational, |x| <= 1/3
    if x < 0:
        return -_atanh(-x)
    y, square, total, n = _fixed(x), _fixed(x * x), 0, 1
    while y:
        total += y // n
        y, n = y * square >> BITS, n + 2
    return total


LN2 = 2 * _atanh(Fraction(1, 3))


def _ln(x):
    x = Fraction(x)
    power = 0
    while x >= Fraction(4, 3):
        x, power = x / 2, power + 1
    while x < Fraction(2, 3):
        x, power = x * 2, power - 1
    return 2 * _atanh((x - 1) / (x + 1)) + power * LN2


def _exp(y):
    power, y = divmod(y, LN2)
    term, total, n = ONE, 0, 1
    while term:
        total += term
        term, n = (term * y >> BITS) // n, n + 1
    return total << power if power >= 0 else total >> -power


def _atan_inverse(n):
    term, total, k, sign = ONE // n, 0, 1, 1
    while term:
        total += sign * (term // k)
        term, k, sign = term // (n * n), k + 2, -sign
    return total


TWO_PI = 8 * (4 * _atan_inverse(5) - _atan_inverse(239))  # Machin


def _expected(dim, base=10000.0, scaling=None, factor=1.0, length=0, low=1.0, high=32.0):
    """Turns a token times 2^BITS."""
    ln = _ln(base)
    if scaling == "base":
        ln += _ln(factor) * dim // (dim - 2)
    turns = [_exp(-2 * i * ln // dim) * ONE // TWO_PI for i in range(dim // 2)]
    if scaling == "linear":
        return [int(t / Fraction(factor)) for t in turns]
    if scaling == "parts":
        stays = [min(max((Fraction(length) * Fraction(t, ONE) - Fraction(low)) / (Fraction(high) - Fraction(low)), 0), 1) for t in turns]
        return [int(t * (s + (1 - s) / Fraction(factor))) for t, s in zip(turns, stays)]
    return turns


PLANS = [dict(dim=128), dict(dim=64, base=500000.0), dict(dim=6, base=10.0), dict(dim=2), dict(dim=1024, base=1e6),
         dict(dim=128, scaling="linear", factor=8.0), dict(dim=40, scaling="linear", factor=0.3),
         dict(dim=128, scaling="base", factor=4.0), dict(dim=4, base=3.7, scaling="base", factor=0.1),
         dict(dim=128, scaling="parts", factor=8.0, length=2048), dict(dim=34, scaling="parts", factor=2.5, length=777, low=0.25, high=9.5),
         dict(dim=8, base=1e-3), dict(dim=8, base=1e-30), dict(dim=8, base=1e300)]


@pytest.mark.parametrize("plan", PLANS, ids=str)
def test_every_bit_of_a_frequency(plan):
    got = [t % (1 << 64) for t in lram.rotary_plan(**plan, device="cpu").turns.tolist()]
    for i, (bits, want) in enumerate(zip(got, _expected(**plan))):
        off = Fraction(want, 1 << BITS - 64) - bits
        off -= round(off / (1 << 64)) * (1 << 64)  # of a whole turn
        assert abs(off) <= Fraction(1, 2) + Fraction(1, 1 << 40), (i, float(off))


def test_what_no_scaling_needs_is_not_read():
    plain = lram.rotary_plan(8, device="cpu").turns.tolist()
    assert lram.rotary_plan(8, factor=None, length=None, low=None, high=None, device="cpu").turns.tolist() == plain
    linear = lram.rotary_plan(8, scaling="linear", factor=2, length=None, low=None, high=None, device="cpu").turns.tolist()
    assert linear == lram.rotary_plan(8, scaling="linear", factor=2.0, device="cpu").turns.tolist()


def test_angles_at_the_farthest_position():
    """What a frequency's rounding leaves of an angle at position 2^31: at most 2^-34 of a turn."""
    got = [t % (1 << 64) for t in lram.rotary_plan(128, device="cpu").turns.tolist()]
    for bits, want in zip(got, _expected(128)):
        assert abs((Fraction(want, ONE) - Fraction(bits, 1 << 64)) * 2 ** 31) <= Fraction(1, 2 ** 34) + Fraction(1, 2 ** 60)


def test_the_series_themselves():
    assert TWO_PI / ONE == 2 * math.pi and _exp(ONE) / ONE == math.e and _ln(10) / ONE == pytest.approx(math.log(10), rel=1e-15)
    assert abs(_exp(_ln(7)) - 7 * ONE) < 1 << 20
