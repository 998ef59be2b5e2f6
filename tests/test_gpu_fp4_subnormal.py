"""What the 4-bit cache holds of values below the type's smallest normal number, bit for bit."""
import pytest
import torch

from oracle import layer_oracle as L

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_subnormal_values(gpu, dt):
    """Blocks of the smallest step, 2^-125, whose borders at 1/4 and values below 1/2 of it are subnormal, alone
    and beside normal values."""
    gen = torch.Generator("cuda").manual_seed(1)
    quarter = 2.0 ** -127
    x = quarter * 4 * torch.rand(64, 32, generator=gen, device="cuda", dtype=torch.float64)
    x[:16] /= 4                                            # all of them subnormal
    near = torch.tensor([0.5, 1.0, 1.0 + 2.0 ** -6, 1.0 - 2.0 ** -6, 1.5, 1.75, 2.0, 3.0, 4.0, 6.0], device="cuda") * quarter
    x[20, :10], x[21, :10] = near, -near
    x[22:24] = 2.0 ** -133
    x[24:26] = 2.0 ** -149
    x[32:48, 0] = 7 * 2.0 ** -125                          # a block of the same step with a normal value
    x[48:, 0] = 1.0                                        # and of a step to which they are nothing
    k = x.to(dt).view(1, 1, 64, 32)
    assert ((k != 0) & (k.abs() < torch.finfo(dt).tiny)).sum() > 500
    cache = gpu.fp4_cache(2, 1, 32, 32)
    table = torch.arange(2, dtype=torch.int32, device="cuda")[None]
    gpu.fp4_cache_write(cache, k, -k, table)
    kr, vr = gpu.fp4_cache_read(cache, table, 64, dtype=torch.float32)
    want = L.held(k)[0]
    assert torch.equal(kr.double(), want) and torch.equal(vr.double(), -want)
