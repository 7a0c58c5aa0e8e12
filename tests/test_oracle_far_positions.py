"""Angles of the oracle of norms and rotation at far positions, against rational numbers."""
import math
from fractions import Fraction

import numpy as np

from oracle import heads as ohead

PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899862803474, 10 ** 89)


def test_angles_of_far_positions_and_large_frequencies():
    positions = np.array([0, 1, -1, 5, 123456789, 2 ** 31 - 1, -2 ** 31])
    frequencies = np.array([1.0, 0.1, 1e-6, 1000.7, 1e9 + 0.1, -2.5, 0.0, 2.0 ** -60, math.pi])
    got = ohead._angle(positions, frequencies)
    for i, p in enumerate(positions):
        for j, f in enumerate(frequencies):
            t = Fraction(int(p)) * Fraction(float(f)) / (2 * PI)
            assert abs(got[i, j] - 2 * math.pi * float(t - round(t))) < 1e-15
    assert np.array_equal(ohead._angle(positions.astype(np.float64), frequencies), got)


def test_near_positions_are_the_product():
    p, f = np.arange(100), 1e4 ** (-np.arange(32) / 32)
    assert np.allclose(np.exp(1j * ohead._angle(p, f)), np.exp(1j * p[:, None] * f), atol=1e-13)
