"""The oracle's angles against rational arithmetic."""
from fractions import Fraction
import math
import random

import pytest
import torch

from oracle import layer_oracle as L
from paper_2207_10284_amd import ops


def inverse_arctan(n, bits=300):
    x = s = (1 << bits) // n
    k, sign = 3, -1
    while x:
        x //= n * n
        s += sign * (x // k)
        k, sign = k + 2, -sign
    return s


TURN = 2 * Fraction(4 * (4 * inverse_arctan(5) - inverse_arctan(239)), 1 << 300)


@pytest.mark.parametrize("where", [0, 1000, 1 << 20, 2 ** 31 - 500, -2 ** 31])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.001])
def test_angles_at_far_positions(where, base):
    """Off by less than 2^-40 where one float64 product would be off by up to 2^-23."""
    assert abs(float(TURN) - 2 * math.pi) < 1e-15
    rng = random.Random(where)
    f = ops.rotary_frequencies(64, base, device="cpu") * 0.99
    p = torch.tensor([where + rng.randrange(0, 499) for _ in range(40)], dtype=torch.int32)
    cos, sin = L.angles(len(p), f, p)
    for i, a in enumerate(p.tolist()):
        for j, b in enumerate(f.tolist()):
            t = Fraction(a) * Fraction(b) / TURN
            t = float((t - round(t)) * TURN)
            assert abs(cos[0, 0, i, j].item() - math.cos(t)) < 2.0 ** -40
            assert abs(sin[0, 0, i, j].item() - math.sin(t)) < 2.0 ** -40
