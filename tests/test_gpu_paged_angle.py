"""The rotary angle modulo a turn, at every position and speed that is taken, against integer arithmetic."""
import math
from fractions import Fraction

import pytest
import torch

from paper_2605_29707_gb300 import binding as b

pytestmark = pytest.mark.gpu
DEV = "cuda"
POSITIONS = [1, -1, 7, 4096, 1 << 20, -(1 << 20), 123456789, -987654321, (1 << 31) - 1, -(1 << 31), 2147483529, 1999999999]
SPEEDS = [1.0, 0.5, 1e-6, 1e-12, 0.9999999, 1.0 / 3, 2e-9, -0.7, math.pi, 6.2831855, 77.7, 511.99997, 1000.123, -1023.9999, 1024.0, -1024.0]


def _inverse_of_two_pi(bits):
    """floor(2^bits / (2 pi)), pi by Machin's formula."""
    wide = bits + 64

    def arctan(x):
        total, term, n, sign = 0, (1 << wide) // x, 1, 1
        while term:
            total, term, n, sign = total + sign * (term // n), term // (x * x), n + 2, -sign
        return total

    pi = 4 * (4 * arctan(5) - arctan(239))
    return (1 << (2 * wide)) // (2 * pi) >> 64


def _cos_sin(p, f):
    """cos and sin of p f: the turn's fraction exact, less its nearest quarter before it becomes a double."""
    turns = Fraction(f) * p * Fraction(_inverse_of_two_pi(320), 1 << 320)
    quarter = math.floor(4 * turns + Fraction(1, 2))
    a = float(turns - Fraction(quarter, 4)) * 2 * math.pi
    c, s = math.cos(a), math.sin(a)
    return [(c, s), (-s, c), (-c, -s), (s, -c)][quarter % 4]


@pytest.mark.parametrize("layout", [b.DOMINO_ROPE_HALF, b.DOMINO_ROPE_PAIRS])
@pytest.mark.parametrize("gradient", [0, 1])
def test_angles(layout, gradient):
    """x = (1, 0) in every pair gives cos and sin.

    Tolerance: the speed in turns is cut at 2^-64, so the angle is off by less than |p| 2^-64 of a turn; the rest after
    the nearest quarter is rounded to fp32 (2^-24, and as much of its sine and cosine or less) and the function is good
    to 2^-23: together below 2^-22 of the result."""
    half = len(SPEEDS)
    pos = torch.tensor(POSITIONS, dtype=torch.int32, device=DEV)
    freq = torch.tensor(SPEEDS, dtype=torch.float32, device=DEV)
    x = torch.zeros((len(POSITIONS), 1, 2 * half), device=DEV)
    i = torch.arange(half, device=DEV)
    i0, i1 = (i, i + half) if layout == b.DOMINO_ROPE_HALF else (2 * i, 2 * i + 1)
    x[..., i0] = 1.0
    y = torch.full_like(x, float("nan"))
    assert b.domino_rope(x, b.DOMINO_F32, 2 * half, 2 * half, pos, freq, 1.0, layout, gradient, len(POSITIONS), 1, 2 * half,
                         2 * half, y, 2 * half, 2 * half, torch.cuda.current_stream()) == 0
    co, si = y[:, 0, i0].double().tolist(), y[:, 0, i1].double().tolist()
    for r, p in enumerate(POSITIONS):
        for j, f in enumerate(freq.double().tolist()):
            c, s = _cos_sin(p, f)
            s = -s if gradient else s
            cut = 2 * math.pi * abs(p) * 2.0 ** -64
            assert abs(co[r][j] - c) <= 2.0 ** -22 * abs(c) + cut, (p, f)
            assert abs(si[r][j] - s) <= 2.0 ** -22 * abs(s) + cut, (p, f)
