"""Exact softmax attention on the GPU against the float64 oracle: both forward
kernels, the gradients, masks, odd sizes, strides, the position bias.

Bounds. u is a type's unit roundoff (bfloat16 2^-8, float32 2^-24), M the sum
of the magnitudes of the terms of a result (the oracle with ``absolute``).
bfloat16, Z: the weights are rounded before the product and enter the row sum
rounded, the result is rounded: 3 u. L: the row sum moves by at most u. dV: P carries L's error (u), is
rounded (u), the result is rounded (u): 3 u. dS: P carries u, delta = G . Z
carries Z's 3 u, the product's two factors together at most 4 u of their magnitudes, its rounding u, the
result's u: 6 u for dQ and dK; dbias sums unrounded dS: 4 u, its result u.
float32: a logit is off by at most e = u (d + 8) max|q||k| scale + 4 u |S| (a
dot product of d terms, the three dropped plane products 2^-23 each, the
exponent's argument), a weight by 2 e + 4 u, each sum of t terms adds (t + 4) u.
Second-order terms: 10%.
"""
import math

import pytest
import torch

from oracle import exact_oracle as E

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(seed, dt, B, H, Hkv, nq, nk, d, layout="bhnd", size=1.0):
    gen = torch.Generator("cuda").manual_seed(seed)

    def rand(h, n):
        shape = (B, n, h, d) if layout == "bnhd" else (B, h, n, d)
        t = (torch.randn(shape, generator=gen, device="cuda") * size).to(DT[dt])
        return t.transpose(1, 2) if layout == "bnhd" else t

    return rand(H, nq), rand(Hkv, nk), rand(Hkv, nk), rand(H, nq)


def options(gpu, seed, B, H, nq, nk, mask="", causal=False, buckets=None, start=False, scale=None, dt="bf16",
            table="same"):
    """The keyword arguments of a call; `mask` a word of l (lengths), k (key mask), e (one batch without keys)."""
    gen = torch.Generator("cuda").manual_seed(seed + 1)
    o = dict(scale=scale, causal=causal)
    if "l" in mask:
        o["lengths"] = torch.randint(0, nk + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    if "k" in mask:
        o["key_mask"] = torch.rand((B, nk), generator=gen, device="cuda") < 0.7
    if "e" in mask and B:
        if "l" in mask:
            o["lengths"][0] = 0
        else:
            o["key_mask"][0] = False
    if start:
        o["q_start"] = torch.randint(-40, nk + 40, (B,), generator=gen, device="cuda", dtype=torch.int32)
    if buckets:
        o["buckets"] = gpu.distance_buckets(*buckets, device="cuda")
        b = torch.randn((buckets[0], H), generator=gen, device="cuda")
        o["bias"] = b if table == "f32" else b.to(DT[dt])
    return o


def slack(q, k, o):
    """What a weight may be off by, relative (float32): 2 e + 4 u, per row."""
    if q.dtype == torch.bfloat16 or 0 in q.shape or 0 in k.shape:
        return torch.zeros(())
    u, d = U[q.dtype], q.shape[3]
    scale = d ** -0.5 if o["scale"] is None else o["scale"]
    big = q.double().norm(dim=3, keepdim=True) * torch.nan_to_num(k.double()).norm(dim=3).max() * scale
    if o.get("bias") is not None:
        big = big + o["bias"].abs().max()
    return 2 * (u * (d + 8) * big + 4 * u * big) + 4 * u


def check_forward(z, lse, q, k, v, o):
    Z, L, P = E.attention(q, k, v, **o)
    M = P @ E._clean(v, o.get("lengths"), o.get("key_mask")).abs().repeat_interleave(q.shape[1] // max(k.shape[1], 1), 1)
    u = U[q.dtype]
    terms = 0 if q.dtype == torch.bfloat16 else (2 * k.shape[2] + 8) * u
    tol = 1.1 * (3 * u + slack(q, k, o).to(M.device) * 2 + terms) * M + 1e-30
    assert not z.isnan().any()
    bad = (z.double() - Z).abs() > tol
    assert not bad.any(), ((z.double() - Z).abs() / tol).max().item()
    empty = L == -math.inf
    assert torch.equal(z[empty], torch.zeros_like(z[empty])) and bool((lse[empty] == -math.inf).all())
    if not bool(empty.all()):
        tl = 1.1 * (u + slack(q, k, o).to(M.device).squeeze(-1) + terms) + 2.0 ** -22 * L.abs()
        assert bool(((lse.double() - L).abs() <= tl)[~empty].all())
    return Z, L, P


def check_gradients(got, q, k, v, g, o, ref=None):
    ref = E.gradients(q, k, v, g, **o) if ref is None else ref
    mag = E.gradients(q, k, v, g, absolute=True, **o)
    u, bf = U[q.dtype], q.dtype == torch.bfloat16
    s = slack(q, k, o).max().item() if q.dtype == torch.float32 and q.numel() and k.numel() else 0.0
    n = max(q.shape[1] * q.shape[2], k.shape[2], 1)
    for name, x, r, m, c in zip(("dq", "dk", "dv", "dbias"), got, ref, mag, (6, 6, 3, 5)):
        if r is None:
            assert x is None
            continue
        t = 0.0 if bf else (4 * n + 4 * q.shape[3]) * u + 4 * s
        if name == "dbias" and not bf:
            t += 4 * s
        tol = 1.1 * (c * (u if bf else 0) + t + U[x.dtype]) * m + 1e-30
        assert x.shape == r.shape and not x.isnan().any(), name
        err = (x.double() - r).abs()
        assert not (err > tol).any(), (name, (err / tol).max().item())


def run(gpu, q, k, v, g, o):
    lse = torch.empty(q.shape[:3], device="cuda")
    z = gpu.exact_attention_forward(q, k, v, lse_out=lse, **o)
    grads = gpu.exact_attention_backward(q, k, v, z, g, lse, **o)
    return z, lse, grads


# dtype, B, H, H_kv, nq, nk, d, layout, options
CASES = [
    ("bf16", 1, 1, 1, 1, 1, 64, "bhnd", {}),
    ("f32", 1, 1, 1, 1, 1, 32, "bhnd", {}),
    ("bf16", 2, 3, 3, 33, 33, 32, "bhnd", {}),
    ("bf16", 2, 4, 2, 65, 129, 64, "bnhd", dict(causal=True)),
    ("f32", 1, 2, 1, 31, 97, 128, "bnhd", dict(causal=True, mask="l")),
    ("f32", 2, 2, 2, 130, 130, 64, "bhnd", dict(mask="k")),
    ("bf16", 3, 2, 1, 100, 260, 128, "bhnd", dict(mask="lke")),
    ("bf16", 2, 2, 2, 150, 64, 64, "bhnd", dict(causal=True)),                       # the first rows have no key
    ("f32", 2, 2, 2, 70, 33, 32, "bnhd", dict(causal=True, start=True, mask="k")),
    ("bf16", 2, 4, 4, 200, 200, 64, "bnhd", dict(buckets=(32, 128, True))),
    ("bf16", 2, 4, 1, 90, 700, 32, "bnhd", dict(buckets=(16, 50, False), causal=True, mask="l")),
    ("f32", 2, 2, 2, 300, 300, 64, "bhnd", dict(buckets=(8, 20, True), mask="ke")),
    ("f32", 1, 4, 2, 65, 513, 128, "bnhd", dict(buckets=(32, 128, True), start=True)),
    ("bf16", 1, 2, 2, 40, 2100, 128, "bhnd", dict(buckets=(64, 256, True), table="f32")),
    ("bf16", 2, 2, 2, 64, 96, 64, "bhnd", dict(scale=1.0)),
    ("f32", 2, 2, 2, 64, 96, 32, "bhnd", dict(scale=0.02)),
    # the shared-tile forward: at least 256 workgroups of 128 rows
    ("bf16", 16, 16, 16, 70, 70, 64, "bnhd", dict(mask="lke")),
    ("bf16", 16, 16, 4, 33, 161, 32, "bhnd", dict(causal=True)),
    ("bf16", 8, 32, 8, 129, 65, 128, "bnhd", dict(mask="k", buckets=(32, 128, True))),
    ("f32", 16, 16, 16, 40, 100, 64, "bnhd", dict(mask="l", buckets=(8, 20, True), causal=True)),
    ("f32", 16, 16, 8, 33, 65, 128, "bhnd", dict(causal=True)),
    ("f32", 16, 16, 8, 50, 129, 32, "bhnd", dict(mask="ke")),
    ("bf16", 2, 128, 128, 160, 100, 32, "bhnd", dict(causal=True, start=True, mask="l")),
    # lengths past one stage of every kernel, and a length that is none
    ("bf16", 1, 2, 2, 513, 1025, 64, "bnhd", dict(causal=True)),
    ("f32", 1, 1, 1, 257, 300, 64, "bnhd", {}),
    ("bf16", 2, 2, 2, 5, 0, 64, "bhnd", {}),
    ("f32", 2, 2, 1, 0, 40, 32, "bhnd", dict(buckets=(8, 20, True))),
    ("bf16", 0, 2, 2, 5, 40, 32, "bhnd", dict(buckets=(8, 20, True))),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_oracle(gpu, case):
    dt, B, H, Hkv, nq, nk, d, layout, opts = CASES[case]
    print("exact", CASES[case], flush=True)
    q, k, v, g = make(100 + case, dt, B, H, Hkv, nq, nk, d, layout)
    o = options(gpu, 200 + case, B, H, nq, nk, dt=dt, **opts)
    z, lse, grads = run(gpu, q, k, v, g, o)
    torch.cuda.synchronize()
    check_forward(z, lse, q, k, v, o)
    check_gradients(grads, q, k, v, g, o)
