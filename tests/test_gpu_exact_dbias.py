"""The bias gradient over many keys on the GPU: sums whose terms cancel."""
import pytest
import torch

from oracle import exact_oracle as E
from tests.test_gpu_exact import make, options, run


@pytest.mark.parametrize("planes,d", [(p, d) for p in (1, 3) for d in (32, 64, 128)])
def test_lds_of_the_dq_pass(planes, d):
    """With the widest window: stages (32 rows where two waves a SIMD or three planes ask for it), the
    bias, four windows of sums, four skewed tiles and eight doubles within 160 KB, the doubles aligned."""
    rows = 64 if (planes == 1 and d < 128) or d == 32 else 32
    for far in (0, 1, 91, 512):
        entries = 2 * far + 128
        before = 4 * planes * rows * d * 2 + 4 * (5 * entries + 4 * 32 * 64)
        assert before % 8 == 0 and before + 64 <= 160 * 1024


@pytest.mark.gpu
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_terms_that_rise_and_fall(gpu, dt):
    """All logits are 0 and G . v_j is a whole number c_j: 1 to 3 over half of 2^20 keys, their negatives
    over the other half, 16 at the ten nearest, so P = 2^-20 and D = P (c_j - 160 P) up to one
    factor of P, and all that is left of the far buckets is -160 P a query.

    Bound, in units of P: a lane's float32 sum reaches 32 tiles x 16 x 3 < 2^11 before it moves to a
    double, each of the 2^16 additions is off by at most 2^-14; a tile's 16 terms stay below 2^6, each
    of the 2^20 additions off by at most 2^-19; the eight workgroups' results below 2^19 by 2^-6 each; D itself, below 4,
    by 2^-22 each: 4 + 2 + 0.13 + 0.25 < 6.5. P, one factor for all: 2^-19 relative. dbias is rounded
    to its type. (A float32 sum over all of a lane's keys would be off by about 60.)"""
    n, d, nq = 1 << 20, 32, 2
    gen = torch.Generator("cuda").manual_seed(1)
    m = n - 200
    c = torch.zeros(n, device="cuda")
    c[:m // 2] = torch.randint(1, 4, (m // 2,), generator=gen, device="cuda").float()
    c[m // 2:m] = -c[:m // 2].flip(0)
    c[-10:] = 16.0
    q = torch.zeros(1, 1, nq, d, dtype=dt, device="cuda")
    k = torch.randn(1, 1, n, d, generator=gen, device="cuda").to(dt)
    v = torch.zeros(1, 1, n, d, dtype=dt, device="cuda")
    v[0, 0, :, 5] = c.to(dt)
    g = torch.zeros_like(q)
    g[..., 5] = 1.0
    o = dict(causal=False, bias=torch.zeros(32, 1, device="cuda"), buckets=gpu.distance_buckets(32, 128, True))
    lse = torch.empty(1, 1, nq, device="cuda")
    z = gpu.exact_attention_forward(q, k, v, lse_out=lse, **o)
    dbias = gpu.exact_attention_backward(q, k, v, z, g, lse, **o)[3]
    ref = E.gradients(q, k, v, g, **o)[3]
    P = 2.0 ** -n.bit_length() * 2
    assert -161 * nq * P < ref[15, 0] < -150 * nq * P
    assert abs(dbias[15, 0].double() - ref[15, 0]) <= nq * 6.5 * P + 2.0 ** -19 * ref[15, 0].abs()


# B, H, H_kv, n_q, n_k, d, what options takes
MANY_KEYS = [
    (1, 1, 1, 64, 20000, 64, dict(buckets=(32, 128, True))),                         # parts of every block
    (2, 2, 1, 256, 9000, 32, dict(buckets=(32, 128, True), mask="lk")),
    (1, 4, 2, 2100, 2100, 128, dict(buckets=(32, 128, False), causal=True)),
    (2, 2, 2, 150, 3000, 64, dict(buckets=(8, 20, True), start=True, mask="k")),
    (3, 8, 8, 333, 1500, 64, dict(buckets=(16, 50, True), mask="le")),
    (1, 2, 2, 31, 12000, 128, dict(buckets=(64, 256, True))),
    (1, 1, 1, 700, 5000, 32, dict(buckets=(4, 8, False), causal=True, mask="l")),
]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(MANY_KEYS)))
def test_bfloat16_over_many_keys(gpu, case):
    """Over many keys the roundings of a bfloat16 Z stay out of dbias (a float32 table: its own
    rounding is 2^-24). What is left in a query's D, 2-norm over the buckets:

    - L is the logarithm of a sum of rounded weights: one factor for the query's D, off by the sum of
      P_ij rho_j, roundings |rho| <= 2^-8, independent: 2^-8 |P_i| is more than twice its root mean
      square, and it meets the query's sums of D by bucket, B_i.
    - float32: the exponent's argument (up to 16: 2^-21), the exponential, two products of up to
      eight matrix steps: 2^-18 of each term, independent over keys: 2^-18 |D_i|.

    2-norms over queries add in quadrature, held to twice their sum. With the roundings of Z it would be about 2^-9 |P_i|
    |G . v| |sums of P by bucket| a query, at least four times the bound except where causal rows of
    few keys outweigh the others."""
    B, H, Hkv, nq, nk, d, opts = MANY_KEYS[case]
    print("many keys", MANY_KEYS[case], flush=True)
    q, k, v, g = make(71 + case, "bf16", B, H, Hkv, nq, nk, d)
    o = options(gpu, 72 + case, B, H, nq, nk, table="f32", **opts)
    assert o["bias"].dtype == torch.float32 and nk > 8 * o["buckets"].numel()
    got = run(gpu, q, k, v, g, o)[2][3]
    ref = E.gradients(q, k, v, g, **o)[3]
    Z, _, P = E.attention(q, k, v, **o)
    V = E._clean(v, o.get("lengths"), o.get("key_mask")).repeat_interleave(H // Hkv, 1)
    dP = g.double() @ V.transpose(2, 3).contiguous()
    D = P * (dP - (g.double() * Z).sum(-1, keepdim=True))
    far = o["buckets"].numel() // 2
    start = torch.full((B,), nk - nq, device="cuda") if o.get("q_start") is None else o["q_start"].long()
    rel = torch.arange(nk, device="cuda") - (start[:, None] + torch.arange(nq, device="cuda"))[:, :, None]
    at = o["buckets"].long()[rel.clamp(-far, far) + far][:, None]
    by_d, by_p = (sum((x * (at == c)).sum(-1).square() for c in range(o["bias"].shape[0])).sqrt() for x in (D, P))
    size = P.norm(dim=-1)
    bound = 2 * ((2.0 ** -8 * size * by_d).norm() + 2.0 ** -18 * D.norm())
    assert (nq == nk and opts["causal"]) or (2.0 ** -9 * (P * dP).norm(dim=-1) * by_p).norm() > 4 * bound
    assert (got.double() - ref).norm() <= bound
