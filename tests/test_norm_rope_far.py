"""Angles of positions so far that 64 bits leave little of a turn, against 60 decimal digits.

A pair's quarter turns are (origin + step * index) * theta^(-2j / d) / (pi / 2) in 64 bits: the frequency is the nearest number to the true one (half a
step, 2^-53 of it), its products with step and origin round once each and so does their sum, 3 steps of 2^-53 of the angle and one more for
the part of the step (indices are small).  The fraction that is left is rounded to 32 bits (half a quarter turn: 2^-26) and goes through the
polynomials and the rotation: 8 * 2^-24 of a unit vector."""
from decimal import Decimal, getcontext

import math

import pytest
import torch

from paper_2609_37001_b200 import binding as B

getcontext().prec = 60


def _pi():
    def arctan_inverse(n):
        x = total = Decimal(1) / n
        k, sign = 1, 1
        while abs(x) > Decimal(10) ** -58:
            x /= n * n
            k, sign = k + 2, -sign
            total += sign * x / k
        return total
    return 4 * (4 * arctan_inverse(5) - arctan_inverse(239))


PI = _pi()


def turns(dims, theta, position):
    """(cos, sin, quarter turns) of every pair at `position` (one exact number an axis)."""
    got = []
    for d, at in zip(dims, position):
        for j in range(d // 2):
            angle = Decimal(at) * (Decimal(theta).ln() * Decimal(-2 * j) / Decimal(d)).exp()
            rest = float(angle.remainder_near(2 * PI))
            got.append((math.cos(rest), math.sin(rest), abs(float(angle / (PI / 2)))))
    return torch.tensor(got, dtype=torch.float64)


def test_reference():
    assert abs(float(PI) - math.pi) == 0
    t = turns((8, 0, 4), 10000, (3, 0, 2))
    want = [3.0 * 10000 ** (-2 * j / 8) for j in range(4)] + [2.0 * 10000 ** (-2 * j / 4) for j in range(2)]
    assert max(abs(float(t[i, 0]) - math.cos(w)) + abs(float(t[i, 1]) - math.sin(w)) for i, w in enumerate(want)) < 1e-14


@pytest.mark.gpu
@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
@pytest.mark.parametrize("dims,theta,origin", [
    ((42, 28, 42), 1000000, (123456789012345, -98765432109876, 111111111111113)),
    ((44, 42, 42), 10000, (123456789012345, 98765432109877, -111111111111113)),
    ((128, 0, 0), 500000, (99999999999999, 0, 0)),
    ((16, 56, 56), 10000, (1000003, 250007, 99999989)),
    ((2, 2, 92), 10000, (0, 17, 100000000003)),
])
def test_far_positions(dims, theta, origin, pairs):
    grid, heads = (2, 3, 4), 2
    rotated = sum(dims)
    x = torch.zeros((heads, 24, 128), device="cuda")
    first = slice(0, rotated, 2) if pairs == "interleaved" else slice(0, rotated // 2)
    second = slice(1, rotated, 2) if pairs == "interleaved" else slice(rotated // 2, rotated)
    x[..., first] = 1.0
    y, _ = B.psa_qk_norm_rope(x, None, grid, dims=dims, theta=float(theta), norm="none", pairs=pairs, origin=origin)
    y = y.cpu().double()
    for n in range(24):
        at = [o + i for o, i in zip(origin, (n // 12, n // 4 % 3, n % 4))]
        want = turns(dims, theta, at)
        limit = 4 * 2.0 ** -53 * want[:, 2] * math.pi / 2 + 8 * 2.0 ** -24
        for h in range(heads):
            assert ((y[h, n, first] - want[:, 0]).abs() <= limit).all() and ((y[h, n, second] - want[:, 1]).abs() <= limit).all()
