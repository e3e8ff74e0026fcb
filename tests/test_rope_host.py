"""How near a rotation's frequencies, fractions of a turn in units of 2^-64, come to those given:
the quotient by 2 pi, in doubles, is off by 2^-53 of itself, and the double nearest 2 pi by 2^-54.5
of that; then the fraction is cut to 64 digits. No call here reaches a kernel."""
import math
from fractions import Fraction

import numpy as np
import pytest


def _pi(digits=80):
    """pi by Machin's formula, in whole numbers."""
    one = 10 ** (digits + 10)

    def arctan(x):
        total = term = one // x
        n, sign = 3, -1
        while term:
            term //= x * x
            total += sign * (term // n)
            n, sign = n + 2, -sign
        return total

    return Fraction(4 * (4 * arctan(5) - arctan(239)), one)


PI = _pi()


def _off(turn, f):
    """|turn - f / (2 pi)| modulo a turn, in turns, and the bound."""
    want = Fraction(float(f)) / (2 * PI)
    d = (Fraction(int(turn), 1 << 64) - want) % 1
    return min(d, 1 - d), abs(want) * Fraction(2) ** -52 + Fraction(1, 1 << 64)


@pytest.mark.parametrize("rot,theta", [(256, 1e6), (96, 5e5), (64, 1e4), (8, 2.0)])
def test_powers_of_theta(jet, rot, theta):
    r = jet.make_rope(rot, theta=theta)
    for i in range(rot // 2):
        d, bar = _off(r.turn[i], math.pow(theta, -2.0 * i / rot))
        assert d <= bar


def test_given_frequencies(jet):
    """Backward ones, too: each is the complement of its forward one."""
    rng = np.random.default_rng(5)
    f = np.concatenate([rng.uniform(-4, 4, 64), 10.0 ** rng.uniform(-12, 6, 64)])
    r = jet.make_rope(256, freq=f)
    for i in range(128):
        d, bar = _off(r.turn[i], f[i])
        assert d <= bar, f[i]
    back = jet.make_rope(256, freq=-f)
    assert all((r.turn[i] + back.turn[i]) % (1 << 64) == 0 for i in range(128))
