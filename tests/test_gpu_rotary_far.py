"""Rotary angles at far positions, for frequencies that are no power of two of a turn.

Rows of ones and zeros give cosine and sine themselves. v = 2^-24. The angle in turns, whose frequency is
split into two float64 values, is off by less than 2^-46; rounded to float32 it is off by at most 2^-26 turns, 2 pi 2^-26
radians; sine and cosine are off by at most 4 units in the last place (2^-22); the products with 1 and the
magnitude and their sum round by v each."""
import pytest
import torch

from oracle import layer_oracle as L

pytestmark = pytest.mark.gpu

BAR = 2.0 ** -22 + 2 * 3.1416 * 2.0 ** -26 + 3 * 2.0 ** -24


def frequencies(gpu, name, r):
    if name == "by_parts":
        return gpu.rotary_frequencies(r, 500000.0, scaling="by_parts", factor=8.0, original=4096)
    if name == "any":
        return torch.rand(r // 2, generator=torch.Generator("cuda").manual_seed(3), device="cuda", dtype=torch.float64) * 2
    return gpu.rotary_frequencies(r, float(name))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("where", ["near", "million", "far", "lowest"])
@pytest.mark.parametrize("freqs", ["10000", "500000", "by_parts", "any"])
def test_cosine_and_sine(gpu, freqs, where, interleaved):
    n, d = 20000, 128
    f = frequencies(gpu, freqs, d)
    lo, hi = {"near": (-1000, 1000), "million": (900000, 1100000), "far": (2 ** 31 - 50000, 2 ** 31 - 1),
              "lowest": (-2 ** 31, -2 ** 31 + 50000)}[where]
    p = torch.randint(lo, hi, (n,), generator=torch.Generator("cuda").manual_seed(5), device="cuda").to(torch.int32)
    x = torch.zeros(1, 1, 1, d, device="cuda")
    a = L.pairs(x, d, interleaved)[0]
    a.fill_(1.0)
    y = gpu.rotary_forward(x.expand(1, 1, n, d), None, f, positions=p, interleaved=interleaved)[0]
    cos, sin = L.angles(n, f, p)
    for got, want in zip(L.pairs(y, d, interleaved), (cos, sin)):
        assert (got.double() - want).abs().max().item() <= BAR


def test_gradients_turn_back_as_far(gpu):
    """The backward at the same positions: a turn there and back gives the row, to two turns' errors of its pair."""
    n, d = 4000, 64
    f = frequencies(gpu, "any", d)
    gen = torch.Generator("cuda").manual_seed(6)
    p = torch.randint(2 ** 31 - 50000, 2 ** 31 - 1, (n,), generator=gen, device="cuda").to(torch.int32)
    x = torch.randn(1, 2, n, d, generator=gen, device="cuda")
    want = L.turn(x, f, p, back=True)
    mag = L.turn(x, f, p, back=True, absolute=True)
    got = gpu.rotary_backward(x, None, freqs=f, positions=p)[0]
    assert bool(((got.double() - want).abs() <= (BAR + 2.0 ** -23) * mag).all())


@pytest.mark.parametrize("where", [0, 2 ** 31 - 70000])
def test_the_angle_is_not_rounded_to_float32(gpu, where):
    """Without the angle's rounding what is left is that of sine and cosine. Errors of a vector (cosine, sine) along its
    turn are the angle's: their mean square over many angles, each off by up to 2^-26 turns, evenly, would be
    (2 pi 2^-26)^2 / 3 for turns of 1/4 to 1/2 alone; the results' rounding, 2^-25 at most, adds less than 2^-50 / 3 along it,
    and sine and cosine, where correct to one unit, at most as much again twice."""
    n, d = 60000, 32
    f = frequencies(gpu, "any", d)
    p = torch.arange(where, where + n, device="cuda").to(torch.int32)
    x = torch.zeros(1, 1, 1, d, device="cuda")
    x[..., : d // 2] = 1.0
    y = gpu.rotary_forward(x.expand(1, 1, n, d), None, f, positions=p)[0].double()
    cos, sin = L.angles(n, f, p)
    along = (y[..., d // 2:] - sin) * cos - (y[..., : d // 2] - cos) * sin
    quarter = cos < 0                                      # turns of 1/4 to 1/2, where float32's are rounded most
    assert along[quarter].square().mean().item() < (2 * 3.1416 * 2.0 ** -26) ** 2 / 3
