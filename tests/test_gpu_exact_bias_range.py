"""Position biases of any size on the GPU: mask values (a key with a bias below
-2^14 does not count), the range of finite ones, rows that carry nothing else.

Bounds. Within the range M = max |bias| sets what the exponent of a weight is off by: the log
normaliser is rounded to float32 and multiplied into other units, as is the logit, and
the gradients subtract one from the other (in dK, dV in a product that may
cut instead of round): at most twelve half steps of numbers up to M log2(e), each at most
2^-24 M log2(e) ln(2), so p = 12 / 2 x 2^-23 M = 12 x 2^-24 M at most. A result carries it at most four times
(its own weight, and delta through Z's weights and their sum); the rest is as
in test_gpu_exact.py.
"""
import math

import pytest
import torch

from oracle import exact_oracle as E
from tests.test_gpu_exact import U, make, run, same, slack

RANGE = 2.0 ** 14


def taken(bias):
    """The table as the operator takes it, float64."""
    b = bias.double()
    return torch.where(b < -RANGE, -math.inf, b.clamp(max=RANGE))


def test_taken():
    b = torch.tensor([-math.inf, -1e9, -16385.0, -16384.0, -3.0, 0.0, 16384.0, 1e9, math.inf])
    assert taken(b).tolist() == [-math.inf] * 3 + [-16384.0, -3.0, 0.0, 16384.0, 16384.0, 16384.0]


def check(z, lse, grads, q, k, v, g, o):
    ref = dict(o, bias=taken(o["bias"]))
    Z, L, P = E.attention(q, k, v, **ref)
    want, mag = E.gradients(q, k, v, g, **ref), E.gradients(q, k, v, g, absolute=True, **ref)
    big = ref["bias"][ref["bias"].isfinite()].abs().max().item() if ref["bias"].isfinite().any() else 0.0
    p, u, bf = 12 * 2.0 ** -24 * big, U[q.dtype], q.dtype == torch.bfloat16
    s = slack(q, k, dict(o, bias=None)).max().item()
    n = max(q.shape[1] * q.shape[2], k.shape[2])
    sums = 0.0 if bf else (4 * n + 4 * q.shape[3]) * u + 4 * s
    M = P @ E._clean(v, o.get("lengths"), o.get("key_mask")).abs().repeat_interleave(q.shape[1] // v.shape[1], 1)
    empty = L == -math.inf
    assert torch.equal(z[empty], torch.zeros_like(z[empty])) and bool((lse[empty] == -math.inf).all())
    for name, x, r, m, c in zip(("z", "dq", "dk", "dv", "dbias"), (z, *grads), (Z, *want), (M, *mag), (3, 6, 6, 3, 5)):
        assert x.isfinite().all(), name
        tol = 1.1 * ((c * u if bf else sums) + 4 * p + U[x.dtype]) * m + 1e-30
        err = (x.double() - r).abs()
        assert not (err > tol).any(), (name, (err / tol).max().item())
    assert bool(((lse.double() - L).abs() <= 1.1 * (u + s + sums) + 2.0 ** -22 * L.abs())[~empty].all())


def table(value, H, dtype, seed):
    """Eight buckets (3 and 7 the outer ones) of four kinds of head: all entries of
    `value`, the outer low one, the near ones, all but the outer high one."""
    gen = torch.Generator("cuda").manual_seed(seed)
    b = torch.randn(8, H, generator=gen, device="cuda")
    jitter = b * (0.0 if abs(value) > RANGE else 1.0)
    for h in range(H):
        rows = [slice(0, 8), [3], [0, 1, 2, 4, 5, 6], slice(0, 7)][h % 4]
        b[rows, h] = value + jitter[rows, h]
    return b.to(dtype)


VALUES = [-1e4, -1.63e4, -1.7e4, -1e9, -1e30, -1e38, -3.3e38, -math.inf, 1e4, 1e9, math.inf]


@pytest.mark.gpu
@pytest.mark.parametrize("dt,d,few,entries", [("bf16", 64, True, "same"), ("bf16", 128, False, "same"), ("bf16", 32, True, "f32"),
                                              ("f32", 64, False, "same"), ("f32", 128, True, "same")])
@pytest.mark.parametrize("value", VALUES)
def test_large_entries(gpu, dt, d, few, entries, value):
    """Rows whose keys all carry the value, near and far ones, and rows with others;
    also with a gradient of zero at the former, as a padded query has."""
    print("bias", dt, d, few, entries, value, flush=True)
    B, H, n = (2, 4, 200) if few else (16, 16, 140)
    q, k, v, g = make(41, dt, B, H, H // 2, n, n, d)
    o = dict(scale=None, causal=False, buckets=gpu.distance_buckets(8, 20, True),
             lengths=torch.tensor([n, 20] * (B // 2), dtype=torch.int32, device="cuda"))
    o["bias"] = table(value, H, torch.float32 if entries == "f32" else q.dtype, 42)
    z, lse, grads = run(gpu, q, k, v, g, o)
    check(z, lse, grads, q, k, v, g, o)
    g[1::2, :, 60:] = 0
    z, lse, grads = run(gpu, q, k, v, g, o)
    check(z, lse, grads, q, k, v, g, o)


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_mask_values_are_one(gpu, dt):
    """Every entry below the range gives the bits of -infinity, every one above it those of its end."""
    q, k, v, g = make(43, dt, 2, 4, 4, 150, 150, 64)
    o = dict(scale=None, causal=True, buckets=gpu.distance_buckets(8, 20, False))
    base = torch.randn(8, 4, device="cuda", generator=torch.Generator("cuda").manual_seed(3)).to(q.dtype)

    def everything(values):
        b = base.clone()
        b[[2, 5, 7]] = torch.tensor(values, device="cuda").to(b.dtype)[:, None]
        z, lse, grads = run(gpu, q, k, v, g, dict(o, bias=b))
        return (z, lse, *grads)

    same(everything([-1e9, -1e5, torch.finfo(q.dtype).min]), everything([-math.inf] * 3))
    same(everything([1e9, 1e5, torch.finfo(q.dtype).max]), everything([RANGE] * 3))
