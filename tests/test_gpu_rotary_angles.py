"""Rotary angles against integers: a frequency is the double that the call gets, position * frequency is reduced to
a fraction of a turn without rounding."""
import math
from fractions import Fraction

import pytest
import torch

import paper_2608_27513_gb300 as damp

pytestmark = pytest.mark.gpu
DEV = "cuda"
BITS = 320


def _pi():
    """pi 2^BITS by Machin's formula, with 32 guard bits."""
    one = 1 << (BITS + 32)

    def arctan_of_inverse(n):
        term = one // n
        total, k = term, 1
        while term:
            term //= -n * n
            k += 2
            total += term // k
        return total

    return (4 * (4 * arctan_of_inverse(5) - arctan_of_inverse(239))) >> 32


def turns(freq, position):
    """position * freq / 2 pi without whole turns, in -1/2 .. 1/2."""
    x = Fraction(freq) * position
    t = (x.numerator << (2 * BITS)) // (x.denominator * 2 * _PI)  # of 2^-BITS turns
    t &= (1 << BITS) - 1
    if t >> (BITS - 1):
        t -= 1 << BITS
    return t / (1 << BITS)


_PI = _pi()


def test_pi():
    assert abs(_PI / 2.0 ** BITS - math.pi) < 1e-15 and _PI.bit_length() == BITS + 2


@pytest.mark.gpu
@pytest.mark.parametrize("positions", [[2**31 - 1 - 17 * i for i in range(600)], [-2**31 + 13 * i for i in range(300)], list(range(1, 300)),
                                       [1 << i for i in range(31)], [131071 + i for i in range(300)]])
@pytest.mark.parametrize("scaling,factor", [("none", 1.0), ("yarn", 8.0)])
def test_angles(positions, scaling, factor):
    """(1, 0) turned is (cos, sin).  The fraction of a turn is held to 2^-64 per position, 2^-33 at 2^31, and to 2^-34
    when it is cut to 32 bits of an eighth of a turn: 2 pi (2^-33 + 2^-34) < 2^-29 radians.  Its FP32 rounding
    is relative to an angle of at most pi/4 (2^-24), and the sine or cosine of that to its value (2^-22): 2^-21."""
    freq, _ = damp.rotary_frequencies(128, base=10000.0, scaling=scaling, factor=factor, device=DEV)
    q = torch.zeros(1, len(positions), 1, 128, device=DEV)
    q[..., :64] = 1.0
    out = damp.rotary(q, None, torch.tensor([positions], dtype=torch.int32, device=DEV), freq)[0][0, :, 0].double().cpu()
    angle = torch.tensor([[2 * math.pi * turns(f, p) for f in freq.tolist()] for p in positions], dtype=torch.float64)
    for got, want in ((out[:, :64], angle.cos()), (out[:, 64:], angle.sin())):
        err = (got - want).abs() - 2.0 ** -21 * want.abs()
        assert err.max().item() < 2.0 ** -29


@pytest.mark.parametrize("freq", [3.0, 1.0, -0.7, 1e-3, 12345.678, 1e-12, 1e-300, 2.0 ** 40 + 0.125, 0.0])
def test_any_frequency(freq):
    positions = [1, 2, 3, -5, 1000, 2**31 - 1, -2**31]
    out = damp.rotary(torch.tensor([1.0, 0.0], device=DEV).repeat(1, len(positions), 1, 1), None,
                      torch.tensor([positions], dtype=torch.int32, device=DEV), torch.tensor([freq], dtype=torch.float64, device=DEV))[0]
    angle = torch.tensor([2 * math.pi * turns(freq, p) for p in positions], dtype=torch.float64)
    for i, want in enumerate((angle.cos(), angle.sin())):
        err = (out[0, :, 0, i].double().cpu() - want).abs() - 2.0 ** -21 * want.abs()
        assert err.max().item() < 2.0 ** -29
