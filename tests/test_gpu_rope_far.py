"""Rotary positions at the farthest positions: sines and cosines good to 2^-24.

Angles come from whole numbers of 200 bits (pi by Machin's formula), so nothing of the expected values is off but by 64-bit sines of reduced angles, 2^-52. The tolerance is that of
test_gpu_rope.py, 6 * 2^-24 * (|a| + |b|) and the half-step of an fp32 result, with no part for the position: an angle is off by 2^-65 turns a token, 2^-34 turns at 2^31, 2^-31 radians.
"""
import os
import sys
from fractions import Fraction

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu
BITS = 200


def arctan_inverse(n):
    """2^BITS * arctan(1 / n), to a few units"""
    total = term = (1 << BITS) // n
    k, sign = 1, 1
    while term:
        term //= n * n
        k, sign = k + 2, -sign
        total += sign * (term // k)
    return total


PI = 4 * (4 * arctan_inverse(5) - arctan_inverse(239))


def reduced(position, frequency):
    """position * frequency modulo 2 pi, -pi .. pi"""
    x = Fraction(float(frequency)) * int(position)
    x = (x.numerator << BITS) // x.denominator % (2 * PI)
    return float(Fraction(x - 2 * PI if x > PI else x, 1 << BITS))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_is_as_good_at_any_position(interleaved):
    from paper_2508_13231_b200 import kvp
    assert abs(PI / 2 ** BITS - np.pi) < 2.0 ** -50
    rng = np.random.default_rng(0)
    positions = np.concatenate(([2 ** 31 - 1, -2 ** 31, -1, 0, 1, 2 ** 30 + 3], rng.integers(-2 ** 31, 2 ** 31, 200))).astype(np.int32)
    for f in (np.array([1.0, 0.7498942093324559, 0.1, 3e-5]), np.array([2.5, -0.3, 6.283185307179586, 1e-9]), np.array([1000.0, -1e-12, 1e6, 0.0]), kvp.rope_frequencies(8, base=5e5)[0].numpy()):
        angle = np.array([[reduced(p, g) for g in f] for p in positions])
        x = rng.standard_normal((len(positions), 2, 8)).astype(np.float32)
        got, _ = kvp.rope(torch.from_numpy(x).cuda(), None, torch.from_numpy(positions).cuda(), torch.from_numpy(f).cuda(), interleaved=interleaved)
        got, x = got.double().cpu().numpy(), x.astype(np.float64)
        one, two = (slice(0, 8, 2), slice(1, 8, 2)) if interleaved else (slice(0, 4), slice(4, 8))
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        both = np.abs(x[..., one]) + np.abs(x[..., two])
        for part, want in ((one, x[..., one] * c - x[..., two] * s), (two, x[..., one] * s + x[..., two] * c)):
            off, room = np.abs(got[..., part] - want), 6 * 2.0 ** -24 * both + 2.0 ** -24 * np.abs(want)
            assert np.all(off <= room), float((off / room).max())
