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
    ("bf16", 4, 16, 16, 300, 520, 64, "bnhd", {}),                                   # stages without a border
    ("bf16", 4, 16, 8, 400, 400, 128, "bnhd", dict(causal=True, mask="l")),
    ("f32", 2, 4, 1, 700, 1100, 64, "bnhd", dict(mask="l", buckets=(32, 128, True))),  # parts of every pass
    ("f32", 1, 4, 2, 600, 600, 32, "bhnd", dict(causal=True)),
    ("bf16", 2, 2, 1, 1500, 1300, 64, "bhnd", dict(causal=True, mask="k")),
    ("bf16", 1, 2, 1, 1100, 1200, 128, "bhnd", dict(buckets=(32, 128, True), causal=True, start=True)),
    ("bf16", 16, 64, 64, 256, 96, 32, "bnhd", dict(causal=True, mask="l")),          # 64 rows a wave
    ("bf16", 8, 64, 64, 512, 300, 64, "bhnd", {}),
    ("bf16", 16, 64, 32, 250, 70, 64, "bhnd", dict(buckets=(8, 20, True), mask="ke")),
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


def pieces(gpu, dt="bf16", seed=3, B=2, H=4, Hkv=2, nq=100, nk=150, d=64, layout="bhnd", **opts):
    q, k, v, g = make(seed, dt, B, H, Hkv, nq, nk, d, layout)
    return q, k, v, g, options(gpu, seed, B, H, nq, nk, dt=dt, **opts)


def same(a, b):
    assert len(a) == len(b)
    for x, y in zip(a, b):
        assert (x is None and y is None) or torch.equal(x, y)


def everything(gpu, q, k, v, g, o):
    z, lse, grads = run(gpu, q, k, v, g, o)
    return (z, lse, *grads)


@pytest.mark.parametrize("dt,nk", [("bf16", 150), ("f32", 150), ("bf16", 2000)])
def test_strides(gpu, dt, nk):
    """Views with dense rows give the bits of their copies: one projection's output
    split in three, rows first, a wider row's part, broadcast batches."""
    print("strides", dt, nk, flush=True)
    q, k, v, g, o = pieces(gpu, dt, nq=nk, nk=nk, H=4, Hkv=4, mask="l", causal=True)
    ref = everything(gpu, q, k, v, g, o)
    B, H, n, d = q.shape
    packed = torch.stack([t.transpose(1, 2) for t in (q, k, v)], 2)          # [B, n, 3, H, d]
    views = [x.transpose(1, 2) for x in packed.unbind(2)]
    assert not views[0].is_contiguous()
    same(everything(gpu, *views, g.transpose(1, 2).contiguous().transpose(1, 2), o), ref)
    first = [t.permute(2, 0, 1, 3).contiguous().permute(1, 2, 0, 3) for t in (q, k, v, g)]   # [n, B, H, d]
    same(everything(gpu, *first, o), ref)
    wide = [torch.cat([t, t.neg()], 3)[..., :d] for t in (q, k, v, g)]
    same(everything(gpu, *wide, o), ref)
    one = [t[:1].expand(B, H, n, d) for t in (q, k, v)]
    same(everything(gpu, *one, g, o), everything(gpu, *(t.contiguous() for t in one), g, o))


@pytest.mark.parametrize("dt,B,H,nq,nk,d,opts", [
    ("bf16", 2, 2, 60, 200, 64, dict(mask="l")), ("f32", 2, 2, 60, 200, 128, dict(mask="k")),
    ("bf16", 16, 16, 40, 150, 64, dict(mask="lk")), ("f32", 16, 16, 40, 150, 32, dict(mask="l", causal=True)),
    ("bf16", 4, 16, 130, 150, 128, dict(mask="k", buckets=(8, 20, True)))])
@pytest.mark.parametrize("junk", [math.nan, math.inf, -3e38])
def test_what_lies_at_masked_keys(gpu, dt, B, H, nq, nk, d, opts, junk):
    """Keys and values that do not count change no bit, and have no gradient."""
    print("masked places", dt, B, nk, d, opts, junk, flush=True)
    q, k, v, g, o = pieces(gpu, dt, B=B, H=H, Hkv=H, nq=nq, nk=nk, d=d, **opts)
    out = torch.zeros(B, nk, dtype=torch.bool, device="cuda")
    if "lengths" in o:
        out |= torch.arange(nk, device="cuda") >= o["lengths"][:, None]
    if "key_mask" in o:
        out |= ~o["key_mask"]
    ref = everything(gpu, q, k, v, g, o)
    k2, v2 = (t.masked_fill(out[:, None, :, None], junk) for t in (k, v))
    got = everything(gpu, q, k2, v2, g, o)
    same(got, ref)
    for t in got[3:5]:
        assert not t.transpose(1, 2)[out].any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("order", ["up", "down", "mixed"])
@pytest.mark.parametrize("few", [True, False])
def test_large_logits(gpu, dt, order, few):
    """Logits of some hundreds that rise along the keys, so that references move
    at many tiles, or fall, so that all but the first tiles vanish."""
    print("large logits", dt, order, few, flush=True)
    B, H = (1, 2) if few else (16, 16)
    q, k, v, g, o = pieces(gpu, dt, B=B, H=H, Hkv=H, nq=64, nk=400, d=64)
    ramp = torch.linspace(0.2, 12.0, 400, device="cuda")
    ramp = {"up": ramp, "down": ramp.flip(0), "mixed": ramp[torch.arange(400, device="cuda") * 7 % 400]}[order]
    k = (k * ramp[:, None] * 4).to(k.dtype)
    z, lse, grads = run(gpu, q, k, v, g, o)
    check_forward(z, lse, q, k, v, o)
    check_gradients(grads, q, k, v, g, o)


def test_bias_of_minus_infinity(gpu):
    """takes its distances out: near and far ones, and all keys of some queries."""
    q, k, v, g, o = pieces(gpu, nq=300, nk=300, buckets=(16, 50, True))
    for gone in ([7], [15], [0, 3, 8], [7, 15], list(range(16))):
        o["bias"] = torch.randn_like(o["bias"])
        o["bias"][gone] = -math.inf
        z, lse, grads = run(gpu, q, k, v, g, o)
        check_forward(z, lse, q, k, v, o)
        check_gradients(grads, q, k, v, g, o)


def test_device_values_out_of_range(gpu):
    """Lengths and starts are taken within their range, bucket entries outside the
    table add nothing and take no gradient."""
    q, k, v, g, o = pieces(gpu, nq=70, nk=90, buckets=(8, 20, True))
    o["lengths"] = torch.tensor([-7, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    ref = dict(o, lengths=torch.tensor([0, 90], dtype=torch.int32, device="cuda"))
    z, lse, grads = run(gpu, q, k, v, g, o)
    check_forward(z, lse, q, k, v, ref)
    check_gradients(grads, q, k, v, g, ref)
    for causal in (False, True):
        o = dict(ref, causal=causal, q_start=torch.tensor([-2 ** 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
        z, lse, grads = run(gpu, q, k, v, g, o)
        check_forward(z, lse, q, k, v, o)
        check_gradients(grads, q, k, v, g, o)
    o = dict(ref, buckets=o["buckets"].clone())
    o["buckets"][::3] = torch.tensor([-1, 8, 2 ** 31 - 1, -2 ** 31, 5], dtype=torch.int32, device="cuda")[
        torch.arange(len(o["buckets"][::3])) % 5]
    z, lse, grads = run(gpu, q, k, v, g, o)
    check_forward(z, lse, q, k, v, o)
    check_gradients(grads, q, k, v, g, o)


def test_no_distances(gpu):
    """far = 0: one entry for every distance, which moves no weight; and a map of one bucket."""
    q, k, v, g, o = pieces(gpu, nq=50, nk=64)
    o["bias"] = torch.randn(3, 4, device="cuda")
    o["buckets"] = torch.tensor([2], dtype=torch.int32, device="cuda")
    z, lse, grads = run(gpu, q, k, v, g, o)
    check_forward(z, lse, q, k, v, o)
    check_gradients(grads, q, k, v, g, o)


def test_outputs_given(gpu):
    """Results go where they are asked for, and nothing beside them changes."""
    q, k, v, g, o = pieces(gpu, nq=97, nk=131, mask="l", buckets=(8, 20, True))
    ref = everything(gpu, q, k, v, g, o)

    def room(t):
        big = torch.full((t.shape[0], t.shape[1] + 1, t.shape[2] + 5, 128), 7.0, dtype=t.dtype, device="cuda")
        return big, big[:, :-1, 2:-3, 32:96]

    bigs, outs = zip(*(room(t) for t in (q, q, k, v)))
    lse = torch.full((2 * 4 * 97 + 64,), 7.0, device="cuda")
    dbias = torch.full((9, 4), 7.0, dtype=q.dtype, device="cuda")
    part = lse[:2 * 4 * 97].view(2, 4, 97)
    z = gpu.exact_attention_forward(q, k, v, out=outs[0], lse_out=part, **o)
    assert z.data_ptr() == outs[0].data_ptr()
    gpu.exact_attention_backward(q, k, v, z, g, part, dq=outs[1], dk=outs[2], dv=outs[3], dbias=dbias[:8], **o)
    same((z, part, outs[1], outs[2], outs[3], dbias[:8]), ref)
    assert bool((lse[2 * 4 * 97:] == 7).all()) and bool((dbias[8] == 7).all())
    for big, out in zip(bigs, outs):
        out.fill_(7.0)
        assert bool((big == 7).all())


def test_refusals(gpu):
    q, k, v, g, o = pieces(gpu, buckets=(8, 20, True))
    ok = dict(o)
    lse = torch.zeros(2, 4, 100, device="cuda")
    bad = [
        (dict(q=q.float()), "k must be a torch.float32"), (dict(k=k[:, :, :-1]), "share shape"),
        (dict(q=q[:, :3]), "multiple of H_kv"), (dict(q=q[0]), "B, heads, n, d"),
        (dict(k=k.transpose(2, 3).contiguous().transpose(2, 3)), "dense rows"),
        (dict(q=torch.empty(2 * 4 * 100 * 64 + 1, device="cuda", dtype=q.dtype)[1:].view(q.shape)), "dense rows"),
        (dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")), "lengths"),
        (dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda")), "lengths"),
        (dict(lengths=torch.zeros(2, dtype=torch.int32)), "lengths"),
        (dict(q_start=torch.zeros(2, 1, dtype=torch.int32, device="cuda")), "q_start"),
        (dict(key_mask=torch.ones(2, 149, dtype=torch.bool, device="cuda")), "key_mask"),
        (dict(key_mask=torch.ones(2, 150, device="cuda")), "key_mask"),
        (dict(key_mask=torch.ones(150, 2, dtype=torch.bool, device="cuda").t()), "key_mask"),
        (dict(bias=None), "go together"), (dict(buckets=None), "go together"),
        (dict(bias=o["bias"].t().contiguous()), "bias"), (dict(bias=o["bias"].half()), "bias"),
        (dict(bias=o["bias"].t().contiguous().t()), "bias"),
        (dict(buckets=o["buckets"][:-1]), "buckets"), (dict(buckets=o["buckets"].long()), "buckets"),
        (dict(out=torch.empty_like(q[:, :, :-1])), "out"), (dict(out=torch.empty_like(q, dtype=torch.float32)), "out"),
        (dict(lse_out=torch.empty(2, 4, 99, device="cuda")), "lse_out"),
    ]
    for change, text in bad:
        a = dict(q=q, k=k, v=v, **ok)
        a.update(change)
        args = [a.pop(n) for n in "qkv"]
        with pytest.raises(ValueError, match=text):
            gpu.exact_attention_forward(*args, **a)
        if "out" not in change and "lse_out" not in change:
            with pytest.raises(ValueError, match=text):
                gpu.exact_attention(*args, **a)
            with pytest.raises(ValueError, match=text):
                gpu.exact_attention_backward(*args, q, g, lse, **a)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        gpu.exact_attention(q.half(), k.half(), v.half())
    for scale in (0.0, -1.0, math.nan):
        with pytest.raises(gpu.MraError, match="MRA_ERR_INVALID_ARG"):
            gpu.exact_attention_forward(q, k, v, scale=scale)
    with pytest.raises(gpu.MraError, match="MRA_ERR_UNSUPPORTED"):
        gpu.exact_attention_forward(*(torch.zeros(1, 1, 8, 48, device="cuda") for _ in range(3)))
    far = torch.zeros(2 * 513 + 1, dtype=torch.int32, device="cuda")
    with pytest.raises(gpu.MraError, match="MRA_ERR_UNSUPPORTED"):
        gpu.exact_attention_forward(q, k, v, bias=o["bias"], buckets=far)
    one = torch.zeros(1, 2, 1, 64, device="cuda", dtype=q.dtype)
    many = torch.zeros(1, 2, 4096, 64, device="cuda", dtype=q.dtype)
    need = gpu.exact_forward_workspace_bytes(one, many, many)
    assert need > 0 and gpu.exact_backward_workspace_bytes(one, many, many) > 0
    with pytest.raises(gpu.MraError, match="MRA_ERR_WORKSPACE"):
        gpu.exact_attention_forward(one, many, many, workspace=torch.empty(need - 256, dtype=torch.uint8, device="cuda"))
    for name in ("dq", "dk", "dv", "dbias"):
        with pytest.raises(ValueError, match=name):
            gpu.exact_attention_backward(q, k, v, q, g, lse, **ok, **{name: torch.empty(1, 1, 1, 64, device="cuda")})
    with pytest.raises(ValueError, match="dbias"):
        gpu.exact_attention_backward(q, k, v, q, g, lse, dbias=o["bias"])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_autograd(gpu, dt):
    """The native node, the Python function and the entry points give the same
    bits; gradients of some inputs only; a gradient of another layout; hooks."""
    print("autograd", dt, flush=True)
    q, k, v, g, o = pieces(gpu, dt, mask="lk", causal=True, buckets=(8, 20, True), layout="bnhd")
    z, lse, grads = run(gpu, q, k, v, g, o)
    bias = o.pop("bias")
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v, bias)]
    native = gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
    python = gpu.ExactAttention.apply(*leaves, o["buckets"], o.get("lengths"), o.get("key_mask"), None, None, True)
    for out in (native, python):
        same((out, *torch.autograd.grad(out, leaves, g)), (z, *grads))
    odd = g.transpose(2, 3).contiguous().transpose(2, 3)
    same(torch.autograd.grad(gpu.exact_attention(*leaves[:3], bias=leaves[3], **o), leaves, odd), grads)
    for n in range(4):
        t = [x.detach() for x in leaves]
        t[n].requires_grad_(True)
        gpu.exact_attention(*t[:3], bias=t[3], **o).backward(g)
        assert torch.equal(t[n].grad, grads[n])
    gpu.exact_attention(*leaves[:3], bias=leaves[3], **o).sum().backward()      # a broadcast gradient
    assert torch.equal(leaves[2].grad, gpu.exact_attention_backward(q, k, v, z, torch.ones_like(g), lse, bias=bias, **o)[2])
    assert not gpu.exact_attention(q, k, v, bias=bias, **o).requires_grad
    with torch.no_grad():
        assert not gpu.exact_attention(*leaves[:3], bias=leaves[3], **o).requires_grad
    seen = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: (seen.append(t.shape), t.cpu())[1], lambda t: t.cuda()):
        out = gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
    same(torch.autograd.grad(out, leaves, g), grads)
    assert len(seen) == 9
    out = gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
    with torch.no_grad():
        leaves[1].add_(1.0)
    with pytest.raises(RuntimeError, match="inplace"):
        out.backward(g)
    plain = [t.clone().requires_grad_(True) for t in (q, k, v)]
    out = gpu.exact_attention(*plain)
    first = torch.autograd.grad(out.float().sum(), plain, create_graph=True)[0]
    assert not first.requires_grad                                             # no second gradient


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_same_bits_every_time(gpu, dt):
    q, k, v, g, o = pieces(gpu, dt, nq=500, nk=900, mask="l", buckets=(32, 128, True))
    ref = everything(gpu, q, k, v, g, o)
    for _ in range(3):
        same(everything(gpu, q, k, v, g, o), ref)


def test_streams(gpu):
    """Two streams at once, each with its own calls, and a backward on its forward's stream."""
    a = pieces(gpu, "bf16", seed=5, nq=300, nk=3000, mask="l", buckets=(32, 128, True))
    b = pieces(gpu, "f32", seed=6, nq=40, nk=2000, causal=True)
    refs = [everything(gpu, *x) for x in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        got = []
        for s, x in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                leaves = [t.clone().requires_grad_(True) for t in x[:3]]
                z = gpu.exact_attention(*leaves, **x[4])
            got.append((z, leaves, x[3]))
        grads = [torch.autograd.grad(z, leaves, g) for z, leaves, g in got]
        torch.cuda.synchronize()
        for ref, (z, _, _), gr in zip(refs, got, grads):
            same((z.detach(), *gr), (ref[0], *ref[2:5]))


@pytest.mark.parametrize("dt,d,nq,nk", [("bf16", 64, 1, 3000), ("f32", 128, 200, 1500), ("bf16", 128, 300, 300)])
def test_in_a_graph(gpu, dt, d, nq, nk):
    """Forward and gradients captured; every replay has the eager bits, with other
    calls in the same workspaces between replays."""
    print("graph", dt, d, nq, nk, flush=True)
    q, k, v, g, o = pieces(gpu, dt, nq=nq, nk=nk, d=d, mask="lk", causal=True, buckets=(8, 20, True))
    other = pieces(gpu, dt, seed=9, nq=nq, nk=nk, d=d)
    ws = torch.empty(max(gpu.exact_forward_workspace_bytes(q, k, v, **o), 1), dtype=torch.uint8, device="cuda")
    bws = torch.empty(gpu.exact_backward_workspace_bytes(q, k, v, **o), dtype=torch.uint8, device="cuda")
    z, lse = torch.empty_like(q), torch.empty(q.shape[:3], device="cuda")
    outs = [torch.empty_like(t) for t in (q, k, v, o["bias"])]

    def work():
        gpu.exact_attention_forward(q, k, v, out=z, lse_out=lse, workspace=ws, **o)
        gpu.exact_attention_backward(q, k, v, z, g, lse, dq=outs[0], dk=outs[1], dv=outs[2], dbias=outs[3],
                                     workspace=bws, **o)

    work()
    torch.cuda.synchronize()
    ref = [t.clone() for t in (z, lse, *outs)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for _ in range(3):
        for t in (z, lse, *outs):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        same((z, lse, *outs), ref)
        gpu.exact_attention_forward(*other[:3], workspace=ws)
        torch.cuda.synchronize()


def test_past_32_bits(gpu):
    """One token against a cache of more than 4 GiB a tensor: the keys that matter lie at its end."""
    n, d = (1 << 24) + 77, 128
    k, v = (torch.zeros(1, 1, n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(1, 2, 1, d, dtype=torch.bfloat16, device="cuda")
    q[0, 0, 0, 3], q[0, 1, 0, 5] = 16.0, 16.0
    k[0, 0, n - 40, 3], k[0, 0, n - 2, 5] = 64.0, 64.0            # logits of 90: all other keys vanish
    v[0, 0, n - 40], v[0, 0, n - 2] = 1.0, 2.0
    z = gpu.exact_attention_forward(q, k, v)
    assert bool((z[0, 0] == 1).all()) and bool((z[0, 1] == 2).all())
    z = gpu.exact_attention_forward(q, k, v, lengths=torch.tensor([n - 39], dtype=torch.int32, device="cuda"))
    assert bool((z[0, 0] == 1).all()) and bool((z[0, 1].float().abs() < 1e-6).all())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_full_budget_of_mra_is_exact(gpu, dt):
    """MRA-2 with every block refined is the attention it approximates, forward and backward."""
    q, k, v, g, _ = pieces(gpu, dt, H=4, Hkv=4, nq=320, nk=320)
    o = dict(scale=None, causal=False)
    a = [t.clone().requires_grad_(True) for t in (q, k, v)]
    mra = gpu.mra_attention(*a, 10)
    exact = gpu.exact_attention(*a)
    for out in (mra, exact):
        Z = E.attention(q, k, v, **o)[0]
        assert (out.double() - Z).abs().max() <= (3.3 * U[DT[dt]] + (1e-5 if dt == "f32" else 0)) * v.abs().max()
        check_gradients((*torch.autograd.grad(out, a, g), None), q, k, v, g, o)


@pytest.mark.parametrize("dt,d,Hkv", [("bf16", 64, 4), ("f32", 32, 2), ("bf16", 128, 1)])
def test_tokens_after_a_prompt(gpu, dt, d, Hkv):
    """A decoder's layer as it serves: a padded prompt in one call, then a token at a
    time against the cache, with a position bias. Every row is the row that one
    call over the whole sequence gives (both within the bounds of the oracle)."""
    print("tokens", dt, d, flush=True)
    B, H, n, new, room = 3, 4, 70, 20, 128
    q, k, v, _ = make(31, dt, B, H, Hkv, n + new, n + new, d, "bnhd")
    o = options(gpu, 31, B, H, 1, 1, buckets=(8, 20, False), dt=dt)
    o["causal"] = True
    prompt = torch.tensor([70, 33, 1], dtype=torch.int32, device="cuda")
    cache = [torch.full((B, room, Hkv, d), math.nan, dtype=DT[dt], device="cuda").transpose(1, 2) for _ in range(2)]
    for c, t in zip(cache, (k, v)):
        c[:, :, :n] = t[:, :, :n]
    whole = E.attention(q, k, v, scale=None, causal=True, bias=o["bias"], buckets=o["buckets"],
                        q_start=torch.zeros(B, dtype=torch.int32, device="cuda"))
    start = torch.zeros(B, dtype=torch.int32, device="cuda")
    z = gpu.exact_attention_forward(q[:, :, :n], *cache, lengths=prompt, q_start=start, **o)
    u = U[DT[dt]]
    M = whole[2] @ v.double().abs().repeat_interleave(H // Hkv, 1)
    tol = 1.1 * (3 * u + (2 * slack(q, k, o) + 400 * u if dt == "f32" else 0)) * M
    for b in range(B):
        m = int(prompt[b])
        assert bool(((z[b, :, :m].double() - whole[0][b, :, :m]).abs() <= tol[b if tol.shape[0] > 1 else 0, :, :m]).all())
    length = prompt.clone()
    rows = torch.arange(B, device="cuda")
    for _ in range(new):
        at = length.long()
        for c, t in zip(cache, (k, v)):
            c.transpose(1, 2)[rows, at] = t.transpose(1, 2)[rows, at]
        length = length + 1
        token = q.transpose(1, 2)[rows, at][:, None].transpose(1, 2)
        z = gpu.exact_attention_forward(token, *cache, lengths=length, q_start=length - 1, **o)
        ref, t = whole[0].transpose(1, 2)[rows, at], tol.transpose(1, 2)[rows, at]
        assert bool(((z[:, :, 0].double() - ref).abs() <= t).all())


def test_results_and_workspaces_refused(gpu):
    """Results whose rows share memory, workspaces elsewhere, sizes past 32 bits."""
    q, k, v, g, o = pieces(gpu)
    z, lse, _ = run(gpu, q, k, v, g, o)
    flat = torch.zeros(1, 1, 1, q.shape[3], device="cuda", dtype=q.dtype)
    with pytest.raises(ValueError, match="out must not be broadcast"):
        gpu.exact_attention_forward(q, k, v, out=flat.expand(q.shape), **o)
    for name, t in (("dq", q), ("dk", k), ("dv", v)):
        with pytest.raises(ValueError, match=f"{name} must not be broadcast"):
            gpu.exact_attention_backward(q, k, v, z, g, lse, **o, **{name: flat.expand(t.shape)})
    size = gpu.exact_backward_workspace_bytes(q, k, v, **o)
    for ws in (torch.empty(size, dtype=torch.uint8), torch.empty(size, 2, dtype=torch.uint8, device="cuda")[:, 0]):
        with pytest.raises(ValueError, match="workspace"):
            gpu.exact_attention_forward(q, k, v, workspace=ws, **o)
        with pytest.raises(ValueError, match="workspace"):
            gpu.exact_attention_backward(q, k, v, z, g, lse, workspace=ws, **o)
    long = torch.zeros(q.shape[0], 1, 1, q.shape[3], device="cuda", dtype=q.dtype).expand(-1, -1, (1 << 32) + 32, -1)
    with pytest.raises(ValueError, match="2\\^31"):
        gpu.exact_attention_forward(q, long, long)
    with pytest.raises(ValueError, match="2\\^31"):
        gpu.exact_attention_backward(q, long, long, z, g, lse)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_bias_held_fixed(gpu, dt):
    """A bias that takes no gradient: the others' gradients have the same bits, near
    and far tiles, one part and several."""
    print("fixed bias", dt, flush=True)
    for nq, nk in ((100, 150), (40, 1300)):
        q, k, v, g, o = pieces(gpu, dt, nq=nq, nk=nk, mask="lk", buckets=(8, 20, True))
        z, lse, grads = run(gpu, q, k, v, g, o)
        leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
        out = gpu.exact_attention(*leaves, **o)
        same((out, *torch.autograd.grad(out, leaves, g)), (z, *grads[:3]))
        assert o["bias"].grad is None and not o["bias"].requires_grad


@pytest.mark.parametrize("dt,d", [("bf16", 64), ("f32", 128)])
def test_autograd_in_a_graph(gpu, dt, d):
    """exact_attention and its backward captured with leaves of their own: every replay
    has the eager bits of the values then in the leaves."""
    print("autograd graph", dt, d, flush=True)
    a = pieces(gpu, dt, nq=200, nk=330, d=d, mask="lk", causal=True, buckets=(8, 20, True))
    b = pieces(gpu, dt, seed=9, nq=200, nk=330, d=d)
    o = dict(a[4])
    tables = o.pop("bias"), torch.flip(a[4]["bias"], (0,))

    def eager(t, table):
        leaves = [x.clone().requires_grad_(True) for x in (*t[:3], table)]
        out = gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
        return [x.detach().clone() for x in (out, *torch.autograd.grad(out, leaves, t[3]))]

    refs = [eager(t, table) for t, table in zip((a, b), tables)]
    leaves = [x.clone().requires_grad_(True) for x in (*a[:3], tables[0])]
    g = a[3].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
        grads = torch.autograd.grad(out, leaves, g)
    for n in (0, 1, 0):
        with torch.no_grad():
            for x, y in zip((*leaves, g), (*(a, b)[n][:3], tables[n], (a, b)[n][3])):
                x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        same((out.detach(), *grads), refs[n])
        eager(b, tables[1])
        torch.cuda.synchronize()
