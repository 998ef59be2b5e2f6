"""How far exact attention is off as a whole: 2-norms of Z and the gradients against
the float64 oracle, which do not grow with a row's length as elementwise bounds do.

float32: the error of a float32 evaluation in plain torch is the measure. The kernels' sums
of plane products cut instead of round, which doubles a step's root mean square, and take six times
the steps, whose errors add up like their root: 2 x 2.45 < FLOAT32 times it. A lost plane or plane product
is outside that (test_lost_products_show).

bfloat16, u = 2^-8: a rounding is off by at most u, 0.42 u in root mean square. Z has two
(weights, result), dV two, dQ and dK three (Z in delta, D, result), dbias one and, below eight keys per
distance of its map, that of Z: in quadrature at most 0.73 u, held to u. A gradient without G . Z is
outside that (test_lost_delta_shows).
"""
import math

import pytest
import torch

from oracle import exact_oracle as E
from tests.test_gpu_exact import U, make, options, run

FLOAT32 = 6.0
NAMES = ("z", "dq", "dk", "dv", "dbias")


def evaluation(q, k, v, g, o, mul=torch.matmul, dtype=torch.float32, delta=True):
    """Z and the gradients in plain torch, products by `mul`, the rest in `dtype`."""
    B, H, nq, d = q.shape
    Hkv, nk = k.shape[1:3]
    scale = d ** -0.5 if o.get("scale") is None else o["scale"]
    K, V = (E._clean(t, o.get("lengths"), o.get("key_mask")).to(dtype).repeat_interleave(H // Hkv, 1) for t in (k, v))
    q, g = q.to(dtype), g.to(dtype)
    none = q[..., :1] * 0.0
    bias, keep = E.logits(none, k[..., :1] * 0.0, 1.0, **{n: x for n, x in o.items() if n != "scale"})
    S = (mul(q, K.mT.contiguous()).to(dtype) * scale + bias.to(dtype)).masked_fill(~keep, -math.inf)
    top = S.amax(-1, keepdim=True)
    P = (S - torch.where(top == -math.inf, 0.0, top)).exp()
    P = P / P.sum(-1, keepdim=True).clamp_min(torch.finfo(dtype).tiny)
    Z = mul(P, V).to(dtype)
    D = mul(g, V.mT.contiguous()).to(dtype)
    D = P * (D - (g * Z).sum(-1, keepdim=True) if delta else D)
    dk, dv = (mul(a.mT.contiguous(), b).to(dtype).unflatten(1, (Hkv, -1)).sum(2) for a, b in ((D, q), (P, g)))
    db = None
    if o.get("bias") is not None:
        far = o["buckets"].numel() // 2
        start = torch.full((B,), nk - nq, device=q.device) if o.get("q_start") is None else o["q_start"].long()
        rel = torch.arange(nk, device=q.device) - (start[:, None] + torch.arange(nq, device=q.device))[:, :, None]
        at = o["buckets"].long()[rel.clamp(-far, far) + far][:, None]
        db = torch.stack([(D * (at == c)).sum((0, 2, 3), dtype=torch.float64) for c in range(o["bias"].shape[0])])
    return Z, mul(D, K).to(dtype) * scale, dk * scale, dv, db


def oracle(q, k, v, g, o):
    return (E.attention(q, k, v, **o)[0], *E.gradients(q, k, v, g, **o))


def ratios(got, q, k, v, g, o):
    """Errors in 2-norm over what they are held to."""
    out = {}
    f32 = q.dtype == torch.float32
    own = evaluation(q, k, v, g, o) if f32 else None
    for n, (name, r) in enumerate(zip(NAMES, oracle(q, k, v, g, o))):
        if r is not None:
            err = (got[n].double() - r).norm()
            out[name] = (err / (FLOAT32 * (own[n].double() - r).norm() if f32 else U[q.dtype] * r.norm())).item()
    return out


# ---------------------------------------------------------------- mistakes show (on the CPU)
def planes(x):
    """hi the upper half of a float32's bits, mid the rest rounded to bfloat16, lo what is left."""
    x = x.float().contiguous()
    hi = (x.view(torch.int32) & -65536).view(torch.float32)
    mid = (x - hi).bfloat16().float()
    return hi, mid, (x - hi - mid).bfloat16().float()


SIX = ((2, 0), (1, 1), (0, 2), (1, 0), (0, 1), (0, 0))


def plane_products(products):
    def mul(a, b):
        pa, pb = planes(a), planes(b)
        return sum(pa[i].double() @ pb[j].double() for i, j in products)
    return mul


def on_cpu(dt, nq, nk, d, bias):
    from paper_2207_10284_amd import ops
    gen = torch.Generator().manual_seed(nq + d)
    q, k, v, g = (torch.randn(1, 2, n, d, generator=gen).to(dt) for n in (nq, nk, nk, nq))
    o = dict(causal=False)
    if bias:
        o.update(bias=torch.randn(32, 2, generator=gen).to(dt), buckets=ops.distance_buckets(32, 128, True, device="cpu"))
    return q, k, v, g, o


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("n", [130, 700])
def test_lost_products_show(d, n):
    """The six plane products are well inside the bound; two planes instead of three, and any one of
    the six missing, are outside it."""
    q, k, v, g, o = on_cpu(torch.float32, n, n, d, True)
    wide = [t.double() for t in (q, k, v, g)]

    def off(products):
        return list(ratios(evaluation(*wide, o, plane_products(products), torch.float64), q, k, v, g, o).values())

    assert max(off(SIX)) < 0.1
    assert min(off(((1, 0), (0, 1), (0, 0)))[:4]) > 4
    for lost in SIX:
        assert min(off([p for p in SIX if p != lost])[:4]) > 1.5, lost


@pytest.mark.parametrize("nq,nk,d", [(130, 130, 64), (40, 2100, 128), (300, 1500, 32)])
def test_lost_delta_shows(nq, nk, d):
    q, k, v, g, o = on_cpu(torch.bfloat16, nq, nk, d, True)
    lost = ratios(evaluation(*(t.double() for t in (q, k, v, g)), o, dtype=torch.float64, delta=False), q, k, v, g, o)
    assert lost["z"] < 1e-6 and lost["dv"] < 1e-6
    assert min(lost["dq"], lost["dk"], lost["dbias"]) > 3


# ---------------------------------------------------------------- on the GPU
# B, H, H_kv, n_q, n_k, d, what options takes
B32 = (32, 128, True)
CASES = [(B, H, Hkv, nq, nk, d, opts)
         for d in (32, 64, 128)
         for B, H, Hkv, nq, nk, opts in (
             (1, 2, 2, 300, 700, dict(buckets=B32)),                                     # few rows: workgroups share keys
             (1, 4, 2, 1, 3000, dict(buckets=(32, 128, False), causal=True)),            # tokens
             (2, 4, 1, 333, 1500, dict(mask="l")),                                       # parts of every pass
             (1, 2, 2, 1503, 1503, dict(buckets=B32)),
             (1, 4, 2, 1100, 1100, dict(causal=True)),
             (16, 16, 8, 200, 200, dict(mask="l")),                                      # blocks that fill the chip
             (8, 12, 12, 512, 512, dict(mask="k", buckets=B32)),
             (8, 64, 64, 512, 300, dict()))]                                             # 64 queries a wave


@pytest.mark.gpu
@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_norms(gpu, dt, case):
    B, H, Hkv, nq, nk, d, opts = CASES[case]
    print("norms", dt, CASES[case], flush=True)
    q, k, v, g = make(500 + case, dt, B, H, Hkv, nq, nk, d)
    o = options(gpu, 600 + case, B, H, nq, nk, dt=dt, **opts)
    z, _, grads = run(gpu, q, k, v, g, o)
    off = ratios((z, *grads), q, k, v, g, o)
    print({n: round(x, 3) for n, x in off.items()}, flush=True)
    assert max(off.values()) <= 1, off


@pytest.mark.gpu
@pytest.mark.parametrize("d", [32, 64, 128])
def test_float32_dbias_of_a_common_part(gpu, d):
    """G . v_j with a large part that all keys share: sums that are cut fall below the exact ones by
    an offset common to a query's keys, which dbias, unlike dQ and dK, would add up over all queries."""
    print("common part", d, flush=True)
    q, k, v, g = make(41, "f32", 1, 2, 2, 1503, 1503, d)
    v, g = v * 0.3 + 1.0, g * 0.3 + 1.0
    o = options(gpu, 42, 1, 2, 1503, 1503, dt="f32", buckets=B32)
    off = ratios((run(gpu, q, k, v, g, o)[0], *run(gpu, q, k, v, g, o)[2]), q, k, v, g, o)
    print({n: round(x, 3) for n, x in off.items()}, flush=True)
    assert off["dbias"] <= 1
