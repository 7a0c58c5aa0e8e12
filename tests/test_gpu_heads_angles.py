"""Rotation by angles of far positions and of frequencies above one, against sines and cosines of angles from whole numbers."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

from nat_testlib import DEV

pytestmark = pytest.mark.gpu
F = 2.0 ** -24
PI = Fraction(314159265358979323846264338327950288419716939937510582097494459230781640628620899862803474, 10 ** 89)


@pytest.fixture(scope="module")
def stage():
    from paper_2603_06619_amd.rollout import RolloutStage
    return RolloutStage(DEV)


def turned(position, frequency):
    t = Fraction(position) * Fraction(frequency) / (2 * PI)
    t = 2 * math.pi * float(t - round(t))
    return math.cos(t), math.sin(t)


NEAR = [2 ** 31 - 1 - 1009 * i for i in range(150)]
FREQUENCIES = [1.0, 0.999999, 0.7310585786300049, 1e-4, 1e-6 * math.e, 3.3, 1000.7, 1e6 + 1 / 3, -2.5, 123456.789, math.pi, 2 * math.pi, 1e-30, 0.0, 1 / 3, 0.1]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("positions", [NEAR, [-p - 1 for p in NEAR], [2 ** 30 + 7 * i * i for i in range(150)], [0, 1, -1, -2 ** 31, 2 ** 31 - 1]])
def test_pairs_of_one_and_zero(stage, positions, interleaved):
    """The rotation of (1, 0) and (0, 1) is the sine and the cosine themselves: the angle's fraction of a turn, below 1/2, is rounded to fp32, which is up to pi F of the
    angle, the functions and the products with 0 and 1 take 4 F more: 8 F."""
    n, R = len(positions), 2 * len(FREQUENCIES)
    pairs = torch.zeros((n, 2, R // 2, 2), device=DEV)
    pairs[:, 0, :, 0] = pairs[:, 1, :, 1] = 1
    x = torch.zeros((n, 2, 64), device=DEV)
    x[..., :R] = (pairs if interleaved else pairs.transpose(-1, -2)).flatten(-2)
    kw = dict(position_ids=torch.tensor(positions, dtype=torch.int32, device=DEV), inv_freq=torch.tensor(FREQUENCIES, dtype=torch.float64, device=DEV), interleaved=interleaved)
    want = np.array([[turned(p, f) for f in FREQUENCIES] for p in positions])
    c, s = want[..., 0], want[..., 1]
    for back, y in ((False, stage.norm_rotate(x, x, **kw)[1]), (True, stage.norm_rotate_backward(x, x, x, x, **kw)[1])):
        y = y[..., :R].double().cpu().numpy()
        a, b = (y[..., 0::2], y[..., 1::2]) if interleaved else (y[..., :R // 2], y[..., R // 2:])
        t = -s if back else s
        for got, ref in ((a[:, 0], c), (b[:, 0], t), (a[:, 1], -t), (b[:, 1], c)):
            assert np.abs(got - ref).max() <= 8 * F, np.unravel_index(np.abs(got - ref).argmax(), ref.shape)
