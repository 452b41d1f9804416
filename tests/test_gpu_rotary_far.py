"""Angles of large frequencies at far positions against exact ones.

Pairs (1, 0) become (cos, sin).  The turns of a frequency are right to 2^-64 and those
of a position to 2^-33, the phase is cut at 2^-32 turns, a rest of an eighth of a turn
and its angle are rounded to 2^-23: under 2^-25 turns in all.  The series and the
products after it: 2^-22."""

import math
from fractions import Fraction

import pytest
import torch

from paper_2606_14782_gb300 import bacon, build

pytestmark = pytest.mark.gpu

FREQUENCIES = [1.0, 4.0, 7.3, 100.0, 402.0, 1000.1, 65536.0, 9.9e5, 1e6, 2 * math.pi, 0.123456789, 1e-12, 0.0, -1.0,
               -3.7, -1e6]
POSITIONS = [0, 1, -1, 12345, 10 ** 9, -2 ** 31, 2 ** 31 - 1, -(2 ** 31 - 1), 2 ** 30 + 7]


def inverse_two_pi():
    """1 / 2 pi to 2^-190, by pi = 16 atan(1/5) - 4 atan(1/239)."""
    one = 1 << 200

    def arctan(x):
        total, term, n = 0, one // x, 1
        while term:
            total += (term // n) * (1 if n % 4 == 1 else -1)
            term, n = term // (x * x), n + 2
        return total

    return Fraction(one, 2 * (16 * arctan(5) - 4 * arctan(239)))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("extra", [0, 2])  # pairs of lanes, and pairs read again
def test_far_angles(interleaved, extra):
    build.build()
    D = 2 * len(FREQUENCIES)
    rotary = bacon.Rotary(D + extra, D, interleaved=interleaved, frequencies=FREQUENCIES)
    x = torch.zeros(len(POSITIONS), 1, D + extra, device="cuda")
    first, second = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    x[..., first] = 1
    y, _ = rotary.apply(x, None, torch.tensor(POSITIONS, dtype=torch.int32, device="cuda"))
    y = y.double().cpu()
    over = inverse_two_pi()
    for i, p in enumerate(POSITIONS):
        for j, theta in enumerate(FREQUENCIES):
            turn = p * Fraction(theta) * over
            angle = math.tau * float(turn - math.floor(turn))
            off = math.tau * 2.0 ** -25 + 2.0 ** -22
            assert abs(y[i, 0, first][j] - math.cos(angle)) <= off, (p, theta)
            assert abs(y[i, 0, second][j] - math.sin(angle)) <= off, (p, theta)
