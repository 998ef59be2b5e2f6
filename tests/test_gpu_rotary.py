"""Rotary positions and head norms on the GPU against the float64 oracle.

Bounds, relative to the magnitudes M of the terms of a result (the oracle with ``absolute``), u the
unit roundoff of its type (bfloat16 2^-8, float32 2^-24), v = 2^-24. An angle of at most half a
turn is rounded to float32 (at most 2^-26 turns, 2^-23.3 radians), sine and cosine
are off by at most 2^-22 more and the magnitude by 2 v, the two products and their sum by 2 v:
2^-21. A norm's mean of d <= 128 squares: its sums are at most 16 + 3 deep, with the square 20 v, the mean
and eps 2 v, halved by the root; root, quotient and two products 5 v: 16 v = 2^-20, so 2^-19 with the
turn. Gradients: g 2^-21, y 2^-20, w g 2^-21 + v, the mean of their products (19 v more) and its product with y, the difference,
the product with r: below 2^-18. A weight's gradient: terms 2^-19, and a float32 sum
of t terms a lane and 128 rows, (t + 130) v.
"""
import pytest
import torch

from oracle import layer_oracle as L

pytestmark = pytest.mark.gpu

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(seed, dt, B, H, Hkv, n, d, layout="bhnd", norm="", wt=None, positions=None):
    gen = torch.Generator("cuda").manual_seed(seed)

    def rand(h):
        shape = (B, n, h, d) if layout == "bnhd" else (B, h, n, d)
        t = torch.randn(shape, generator=gen, device="cuda").to(DT[dt])
        return t.transpose(1, 2) if layout == "bnhd" else t

    q, gq = rand(H), rand(H)
    k, gk = (rand(Hkv), rand(Hkv)) if Hkv else (None, None)
    w = {s: (1 + 0.3 * torch.randn(d, generator=gen, device="cuda")).to(DT[wt or dt]) if s in norm else None for s in "qk"}
    p = None
    if positions == "n":
        p = torch.randint(-50, 5000, (n,), generator=gen, device="cuda", dtype=torch.int32)
    elif positions == "bn":
        p = torch.randint(0, 1 << 20, (B, n), generator=gen, device="cuda", dtype=torch.int32)
    elif positions == "far":
        p = torch.randint(2 ** 31 - 5000, 2 ** 31 - 1, (B, n), generator=gen, device="cuda").to(torch.int32)
    elif positions == "shared":
        p = torch.arange(7, 7 + n, device="cuda", dtype=torch.int32).expand(B, n)
    return q, k, gq, gk, w["q"], w["k"], p


def held_to(x, ref, mag, rel, name):
    assert x.shape == ref.shape and not x.isnan().any(), name
    tol = U[x.dtype] * ref.abs() * 1.01 + rel * mag + 1e-37
    err = (x.double() - ref).abs()
    assert not (err > tol).any(), (name, (err / tol).max().item())


def check(q, k, wq, wk, freqs, p, results, grads=None, gq=None, gk=None, interleaved=False, magnitude=1.0, eps=1e-6):
    kw = dict(positions=p, interleaved=interleaved, magnitude=magnitude)
    for i, (x, w, name) in enumerate(((q, wq, "q"), (k, wk, "k"))):
        if x is None:
            assert results[i] is None
            continue
        rel = 2.0 ** -19 if w is not None else 2.0 ** -21
        held_to(results[i], L.rotary(x, freqs, w, eps, **kw), L.rotary(x, freqs, w, eps, absolute=True, **kw), rel, name)
        if grads is None:
            continue
        g = gq if i == 0 else gk
        dx, dw = L.rotary_grads(g, x, freqs, w, eps, **kw)
        mx, mw = L.rotary_grads(g, x, freqs, w, eps, absolute=True, **kw)
        held_to(grads[i], dx, mx, 2.0 ** -18 if w is not None else 2.0 ** -21, "d" + name)
        if w is None:
            assert grads[2 + i] is None
        else:
            rows = x.shape[0] * x.shape[1] * x.shape[2]
            held_to(grads[2 + i], dw, mw, 2.0 ** -19 + (rows / 32 + 130) * 2.0 ** -24, f"d{name}_weight")


# dtype, B, H, H_kv, n, d, rot, layout, interleaved, norm, weights' dtype, positions, magnitude
CASES = [
    ("bf16", 1, 1, 1, 1, 64, 64, "bhnd", False, "", None, None, 1.0),
    ("f32", 1, 1, 0, 1, 32, 32, "bhnd", True, "q", None, "n", 1.0),
    ("bf16", 32, 12, 12, 1, 64, 64, "bnhd", False, "", None, "bn", 1.0),
    ("bf16", 2, 3, 1, 33, 128, 128, "bnhd", False, "qk", None, "bn", 1.2),
    ("f32", 2, 4, 2, 31, 128, 64, "bhnd", True, "", None, "far", 1.0),
    ("f32", 3, 5, 5, 70, 64, 16, "bnhd", False, "qk", None, "n", 0.5),
    ("bf16", 3, 5, 1, 70, 64, 48, "bhnd", False, "q", "f32", "bn", 1.0),
    ("bf16", 2, 2, 2, 129, 32, 16, "bnhd", True, "k", None, "shared", 1.0),
    ("bf16", 2, 6, 3, 65, 128, 112, "bhnd", True, "qk", "f32", None, 1.0),
    ("f32", 1, 2, 2, 1000, 32, 0, "bnhd", False, "qk", None, None, 1.0),
    ("bf16", 2, 4, 4, 700, 64, 64, "bhnd", False, "qk", None, "far", 1.35),
    ("bf16", 1, 1, 8, 300, 32, 32, "bnhd", False, "qk", None, None, 1.0),
    ("f32", 1, 16, 4, 4100, 128, 128, "bnhd", False, "qk", None, "bn", 1.0),          # tiles of 16, several a workgroup
    ("bf16", 2, 3, 3, 9001, 64, 32, "bhnd", True, "qk", None, None, 1.0),
    ("bf16", 700, 2, 1, 13, 32, 32, "bnhd", False, "", None, "bn", 1.0),
    ("f32", 5, 0, 3, 40, 64, 64, "bhnd", False, "k", None, None, 1.0),                # no queries at all
    ("bf16", 0, 4, 2, 9, 64, 64, "bhnd", False, "qk", None, None, 1.0),
    ("bf16", 2, 4, 2, 0, 64, 64, "bhnd", False, "qk", "f32", "bn", 1.0),
]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_against_the_oracle(gpu, case):
    dt, B, H, Hkv, n, d, rot, layout, inter, norm, wt, positions, mag = CASES[case]
    print("rotary", CASES[case], flush=True)
    q, k, gq, gk, wq, wk, p = make(300 + case, dt, B, H, Hkv, n, d, layout, norm, wt, positions)
    freqs = gpu.rotary_frequencies(rot) if rot else None
    kw = dict(positions=p, interleaved=inter, magnitude=mag, q_weight=wq, k_weight=wk)
    results = gpu.rotary_forward(q, k, freqs, **kw)
    grads = gpu.rotary_backward(gq, gk, q, k, freqs, **kw)
    torch.cuda.synchronize()
    check(q, k, wq, wk, freqs, p, results, grads, gq, gk, inter, mag)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["", "q", "qk"])
def test_autograd(gpu, dt, norm):
    """The native node and the Python function give the bits of the direct calls."""
    q, k, gq, gk, wq, wk, p = make(5, dt, 2, 4, 2, 77, 64, "bnhd", norm, None, "bn")
    freqs = gpu.rotary_frequencies(32)
    kw = dict(positions=p, magnitude=1.1)
    y = gpu.rotary_forward(q, k, freqs, q_weight=wq, k_weight=wk, **kw)
    want = gpu.rotary_backward(gq, gk, q, k, freqs, q_weight=wq, k_weight=wk, **kw)
    leaves = [None if t is None else t.detach().clone().requires_grad_(True) for t in (q, k, wq, wk)]
    given = [t for t in leaves if t is not None]
    native = gpu.rotary(leaves[0], leaves[1], freqs, q_weight=leaves[2], k_weight=leaves[3], **kw)
    python = gpu.Rotary.apply(*leaves, freqs, p, False, 1.1, 1e-6)
    for z in (native, python):
        assert torch.equal(z[0], y[0]) and torch.equal(z[1], y[1])
        got = torch.autograd.grad(z, given, (gq, gk))
        for a, b in zip(got, [w for w in want if w is not None]):
            assert torch.equal(a, b)
    # one result alone, and q alone
    for call in (lambda: gpu.rotary(leaves[0], leaves[1], freqs, q_weight=leaves[2], k_weight=leaves[3], **kw),
                 lambda: gpu.Rotary.apply(*leaves, freqs, p, False, 1.1, 1e-6)):
        got = torch.autograd.grad(call()[1], given, gk, allow_unused=True)
        assert got[0] is None and torch.equal(got[1], want[1])
    alone = gpu.rotary(leaves[0], None, freqs, q_weight=leaves[2], **kw)
    assert alone[1] is None
    assert torch.equal(torch.autograd.grad(alone[0], leaves[0], gq)[0], want[0])


def test_gradients_against_differences(gpu):
    """A directional derivative of the float32 call by central differences; step 2^-8 leaves a
    relative h^2 of its third derivative and 2^-24 / h of rounding."""
    q, k, gq, gk, wq, wk, p = make(9, "f32", 1, 2, 2, 9, 32, "bhnd", "qk", None, "n")
    freqs = gpu.rotary_frequencies(32)
    kw = dict(positions=p)
    dq, dk, dwq, dwk = gpu.rotary_backward(gq, gk, q, k, freqs, q_weight=wq, k_weight=wk, **kw)
    gen = torch.Generator("cuda").manual_seed(1)
    dirs = [torch.randn(t.shape, generator=gen, device="cuda") for t in (q, k, wq, wk)]
    h = 2.0 ** -8

    def loss(s):
        a, b, c, e = (t + s * h * u for t, u in zip((q, k, wq, wk), dirs))
        yq, yk = gpu.rotary_forward(a, b, freqs, q_weight=c, k_weight=e, **kw)
        return ((yq.double() * gq).sum() + (yk.double() * gk).sum()).item()

    slope = (loss(1) - loss(-1)) / (2 * h)
    want = sum((g.double() * u).sum().item() for g, u in zip((dq, dk, dwq, dwk), dirs))
    size = sum((g.double() * u).abs().sum().item() for g, u in zip((dq, dk, dwq, dwk), dirs))
    assert abs(slope - want) <= 1e-3 * size


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
@pytest.mark.parametrize("norm", ["", "qk"])
def test_in_place(gpu, layout, norm):
    q, k, gq, gk, wq, wk, p = make(6, "bf16", 3, 4, 2, 50, 128, layout, norm, None, "bn")
    freqs = gpu.rotary_frequencies(64)
    kw = dict(positions=p, q_weight=wq, k_weight=wk)
    y = gpu.rotary_forward(q, k, freqs, **kw)
    grads = gpu.rotary_backward(gq, gk, q, k, freqs, **kw)
    a, b = gq.clone(), gk.clone()
    got = gpu.rotary_backward(a, b, q, k, freqs, dq=a, dk=b, **kw)
    assert got[0].data_ptr() == a.data_ptr() and torch.equal(a, grads[0]) and torch.equal(b, grads[1])
    z = gpu.rotary_forward(q, k, freqs, q_out=q, k_out=k, **kw)
    assert z[0].data_ptr() == q.data_ptr() and torch.equal(q, y[0]) and torch.equal(k, y[1])


def test_strides(gpu):
    """Views of one projection's output, broadcast heads and batches, rows of a wider tensor."""
    gen = torch.Generator("cuda").manual_seed(3)
    qkv = torch.randn(2, 45, 3, 4, 64, generator=gen, device="cuda").to(torch.bfloat16)
    q, k, _ = (t.transpose(1, 2) for t in qkv.unbind(2))
    freqs = gpu.rotary_frequencies(64)
    wide = torch.zeros(2, 4, 45, 192, device="cuda", dtype=torch.bfloat16)
    y = gpu.rotary_forward(q, k, freqs, q_out=wide[..., 64:128])
    check(q, k, None, None, freqs, None, y)
    assert not wide[..., :64].any() and not wide[..., 128:].any()
    one = torch.randn(1, 1, 45, 64, generator=gen, device="cuda")
    y = gpu.rotary_forward(one.expand(3, 4, 45, 64), one.expand(3, 2, 45, 64), freqs)
    check(one.expand(3, 4, 45, 64), one.expand(3, 2, 45, 64), None, None, freqs, None, y)
    g = torch.randn(1, 1, 1, 64, generator=gen, device="cuda").expand(3, 4, 45, 64)
    x = torch.randn(3, 4, 45, 64, generator=gen, device="cuda", requires_grad=True)
    z, _ = gpu.rotary(x, None, freqs)
    assert torch.equal(torch.autograd.grad(z, x, g)[0], gpu.rotary_backward(g.contiguous(), None, freqs=freqs)[0])


def test_far_positions_are_as_exact_as_near_ones(gpu):
    """Position p + T where T frequency is a whole number of turns gives position p."""
    freqs = torch.full((16,), 2 * torch.pi / 1024, dtype=torch.float64, device="cuda")
    x = torch.randn(1, 1, 200, 32, device="cuda")
    near = torch.arange(200, device="cuda", dtype=torch.int32)
    a = gpu.rotary_forward(x, None, freqs, positions=near)[0]
    b = gpu.rotary_forward(x, None, freqs, positions=near + 1024 * 2000000)[0]
    assert (a - b).abs().max() <= 2.0 ** -21 * 2 * x.abs().max()


def test_strides_past_32_bits(gpu):
    """Heads and batches that begin past 2^32 bytes, read and written."""
    big = torch.empty(5 << 30, dtype=torch.uint8, device="cuda").view(torch.bfloat16)
    x = big.as_strided((2, 2, 40, 64), ((1 << 31) + 64 * 64, 64 * 80, 64, 1))
    y = big.as_strided((2, 2, 40, 64), ((1 << 31) + 64 * 64, 64 * 80, 64, 1), 64 * 40)
    gen = torch.Generator("cuda").manual_seed(2)
    x.copy_(torch.randn(2, 2, 40, 64, generator=gen, device="cuda"))
    y.zero_()
    freqs = gpu.rotary_frequencies(64)
    out = gpu.rotary_forward(x, None, freqs, q_out=y)
    check(x, None, None, None, freqs, None, out)
    assert torch.equal(gpu.rotary_backward(x, None, freqs=freqs, dq=y)[0],
                       gpu.rotary_backward(x.contiguous(), None, freqs=freqs)[0])


def test_repeats_are_the_same_bits(gpu):
    q, k, gq, gk, wq, wk, p = make(8, "bf16", 2, 8, 2, 3000, 64, "bnhd", "qk", None, "bn")
    freqs = gpu.rotary_frequencies(64)
    first = gpu.rotary_backward(gq, gk, q, k, freqs, positions=p, q_weight=wq, k_weight=wk)
    for _ in range(3):
        again = gpu.rotary_backward(gq, gk, q, k, freqs, positions=p, q_weight=wq, k_weight=wk)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_stream_and_graph(gpu):
    q, k, gq, gk, wq, wk, p = make(11, "bf16", 2, 4, 2, 300, 64, "bhnd", "qk", None, "bn")
    freqs = gpu.rotary_frequencies(64)
    leaves = [t.detach().clone().requires_grad_(True) for t in (q, k, wq, wk)]

    def step():
        z = gpu.rotary(leaves[0], leaves[1], freqs, positions=p, q_weight=leaves[2], k_weight=leaves[3])
        return (*(t.detach() for t in z), *torch.autograd.grad(z, leaves, (gq, gk)))

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del got
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step()
    for seed in range(3):
        fresh = make(20 + seed, "bf16", 2, 4, 2, 300, 64, "bhnd", "qk", None, "bn")
        with torch.no_grad():
            for t, x in zip(leaves, (fresh[0], fresh[1], fresh[4], fresh[5])):
                t.copy_(x)
        p.copy_(fresh[6])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed
        del want


def test_differentiated_once(gpu):
    q, k, gq, gk, wq, wk, p = make(12, "f32", 1, 2, 2, 20, 32, "bhnd", "q")
    freqs = gpu.rotary_frequencies(32)
    q.requires_grad_(True)
    for call in (lambda: gpu.rotary(q, k, freqs, q_weight=wq)[0],
                 lambda: gpu.Rotary.apply(q, k, wq, None, freqs, None, False, 1.0, 1e-6)[0]):
        g = torch.ones_like(q).requires_grad_(True)
        (dq,) = torch.autograd.grad(call(), q, g, create_graph=True)
        with pytest.raises(RuntimeError, match="differentia"):
            torch.autograd.grad(dq.sum(), g)
        with pytest.warns(UserWarning, match="not differentiable"):
            torch.autograd.grad(call(), q, torch.ones_like(q), create_graph=True)


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("which", ["q", "q_weight"])
def test_a_captured_backward_with_an_eager_graph_alive_is_refused(gpu, path, which):
    """The refusal alone is called, inside captures of forward calls: no such backward is run."""
    q, k, _, _, wq, wk, p = make(13, "bf16", 2, 4, 2, 30, 64, norm="qk")
    freqs = gpu.rotary_frequencies(64)
    tensors = dict(q=q, k=k, q_weight=wq, k_weight=wk)
    leaf = tensors[which] = tensors[which].clone().requires_grad_(True)

    def forward():
        t = [tensors[n] for n in ("q", "k", "q_weight", "k_weight")]
        if path == "native":
            return gpu.rotary(t[0], t[1], freqs, q_weight=t[2], k_weight=t[3])[0]
        return gpu.Rotary.apply(*t, freqs, None, False, 1.0, 1e-6)[0]

    def captured():
        graph, error = torch.cuda.CUDAGraph(), None
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            try:
                z = forward()
                gpu.bind_layer().check_capture(z)
                del z
            except RuntimeError as e:
                error = str(e)
        return error

    assert captured() is None
    eager = leaf * 2.0
    assert "eager graph" in captured()
    gpu.bind_layer().check_capture(forward())      # not captured: nothing to refuse
    del eager
    assert captured() is None


def test_refusals(gpu):
    q, k, gq, gk, wq, wk, p = make(14, "bf16", 2, 4, 2, 30, 64, norm="qk", positions="bn")
    freqs = gpu.rotary_frequencies(64)
    for bad, match in ((dict(k=k[:1]), "share"), (dict(k=k.float()), "k must be"), (dict(k=k[..., :32]), "share"),
                       (dict(freqs=freqs.float()), "freqs"), (dict(freqs=freqs[:4]), "freqs"),
                       (dict(freqs=gpu.rotary_frequencies(128)), "freqs"), (dict(freqs=freqs.cpu()), "freqs"),
                       (dict(positions=p.long()), "positions"), (dict(positions=p[:1]), "positions"),
                       (dict(positions=p.t()), "positions"), (dict(q_weight=wq[:32]), "q_weight"),
                       (dict(k_weight=wk.half()), "k_weight"), (dict(q_weight=wq.float()), "share their dtype"),
                       (dict(q=q.transpose(2, 3)), "dense rows|share"), (dict(k=None), "k_weight without k"),
                       (dict(q_out=q[:1].expand_as(q)), "broadcast")):
        a = dict(q=q, k=k, freqs=freqs, positions=p, q_weight=wq, k_weight=wk)
        a.update(bad)
        with pytest.raises(ValueError, match=match):
            gpu.rotary_forward(a.pop("q"), a.pop("k"), a.pop("freqs"), **a)
    with pytest.raises(TypeError, match="float16|Half"):
        gpu.rotary(q.half(), None, freqs)
    for bad in (dict(eps=0.0), dict(eps=-1.0), dict(magnitude=float("inf"))):
        with pytest.raises(gpu.MraError, match="INVALID"):
            gpu.rotary(q, k, freqs, q_weight=wq, **bad)
    with pytest.raises(ValueError, match="q is needed"):
        gpu.rotary_backward(gq, gk, freqs=freqs, q_weight=wq)
    with pytest.raises(ValueError, match="go with"):
        gpu.rotary_backward(gq, None, freqs=freqs, dk=gk)
