"""The ways into ops.rotary: plain tensors take the native node, others the Python function; what neither can do is
refused. And its backward where a workgroup takes several tiles of tokens."""
import pytest
import torch

from oracle import layer_oracle as L
from tests.test_gpu_rotary import check, make

pytestmark = pytest.mark.gpu


class _Tagged(torch.Tensor):
    pass


def inputs(gpu, dt="f32"):
    q, k, gq, gk, wq, wk, p = make(31, dt, 2, 4, 2, 33, 64, norm="qk", positions="bn")
    return q, k, gq, gk, wq, wk, p, gpu.rotary_frequencies(64)


def test_which_path(gpu):
    q, k, _, _, wq, wk, p, freqs = inputs(gpu)
    x = q.clone().requires_grad_(True)
    for t in (x, torch.nn.Parameter(q)):
        y = gpu.rotary(t, k, freqs, positions=p, q_weight=wq, k_weight=wk)
        assert type(y[0]) is torch.Tensor and "RotaryBackward" not in type(y[0].grad_fn).__name__
    tagged = x.detach().as_subclass(_Tagged).requires_grad_(True)
    y = gpu.rotary(tagged, k, freqs, positions=p, q_weight=wq, k_weight=wk)
    assert "RotaryBackward" in type(y[0].grad_fn).__name__


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_tensor_subclass_gets_its_own_type(gpu, dt):
    q, k, gq, gk, wq, wk, p, freqs = inputs(gpu, dt)
    kw = dict(positions=p)
    want = gpu.rotary_forward(q, k, freqs, q_weight=wq, k_weight=wk, **kw)
    back = gpu.rotary_backward(gq, gk, q, k, freqs, q_weight=wq, k_weight=wk, **kw)
    t = [x.clone().as_subclass(_Tagged) for x in (q, k, wq, wk)]
    for call in (gpu.rotary_forward, gpu.rotary):
        got = call(t[0], t[1], freqs, q_weight=t[2], k_weight=t[3], **kw)
        for a, b in zip(got, want):
            assert type(a) is _Tagged and torch.equal(a.as_subclass(torch.Tensor), b)
        assert call(t[0], None, freqs, **kw)[1] is None
    leaves = [x.requires_grad_(True) for x in t]
    y = gpu.rotary(leaves[0], leaves[1], freqs, q_weight=leaves[2], k_weight=leaves[3], **kw)
    for a, b in zip(torch.autograd.grad(y, leaves, (gq, gk)), back):
        assert torch.equal(a.as_subclass(torch.Tensor), b)


def test_traced(gpu):
    """Under torch.jit.trace the Python function runs; its values are those of the call."""
    q, k, _, _, wq, wk, p, freqs = inputs(gpu)
    seen = []

    def f(a):
        seen.append(torch._C._get_tracing_state() is not None)
        return gpu.rotary(a, k, freqs, positions=p, q_weight=wq, k_weight=wk)[0]

    g = torch.jit.trace(f, q, check_trace=False)
    assert seen == [True]
    assert torch.equal(g(q), f(q))


def test_transforms_and_forward_mode_are_refused(gpu):
    q, k, _, _, wq, wk, p, freqs = inputs(gpu)
    cache = gpu.fp4_cache(4, 2, 32, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lengths = torch.full((2,), 20, dtype=torch.int32, device="cuda")
    for call in (lambda a: gpu.rotary(a, k, freqs, positions=p, q_weight=wq, k_weight=wk)[0],
                 lambda a: gpu.rotary(a, None, freqs)[0],
                 lambda a: gpu.rotary_forward(a, None, freqs)[0],
                 lambda a: gpu.rotary_backward(a, None, freqs=freqs)[0],
                 lambda a: gpu.fp4_cache_attention(a, cache, table, lengths)):
        with pytest.raises(RuntimeError):
            torch.func.vmap(call)(q.expand(2, *q.shape))
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(q, torch.ones_like(q))
        with pytest.raises(RuntimeError):
            gpu.rotary(dual, k, freqs, positions=p, q_weight=wq, k_weight=wk)
    with pytest.raises(RuntimeError):
        torch.func.grad(lambda a: gpu.rotary(a, None, freqs)[0].sum())(q)


# more than 1024 tiles of eight tokens, so that a workgroup of the backward takes several
@pytest.mark.parametrize("dt,B,H,Hkv,n,d,rot,inter,wt", [
    ("f32", 1, 3, 1, 20011, 128, 128, False, None), ("bf16", 2, 4, 2, 12007, 128, 64, False, "f32"),
    ("bf16", 1, 2, 2, 33001, 32, 32, True, None), ("f32", 2, 2, 1, 9001, 64, 48, True, None),
])
def test_backward_over_several_tiles(gpu, dt, B, H, Hkv, n, d, rot, inter, wt):
    q, k, gq, gk, wq, wk, p = make(41, dt, B, H, Hkv, n, d, "bnhd", "qk", wt, "bn")
    freqs = gpu.rotary_frequencies(rot)
    kw = dict(positions=p, interleaved=inter, q_weight=wq, k_weight=wk)
    results = gpu.rotary_forward(q, k, freqs, **kw)
    grads = gpu.rotary_backward(gq, gk, q, k, freqs, **kw)
    check(q, k, wq, wk, freqs, p, results, grads, gq, gk, inter)
    # A tile's eight tokens lost or taken twice are at least 8 of T rows, 1.5% of the sum's size (which grows like the root of
    # T) in the mean over its elements; the bound above goes by the sum of magnitudes, some 0.64 T. Terms within 2^-19 and
    # float32 sums of below 64 + 130 terms are off by at most (2^-19 + 194 2^-24) 0.64 T, 0.3% of that size at T = 66002.
    for i, (x, w, g) in enumerate(((q, wq, gq), (k, wk, gk))):
        dw = L.rotary_grads(g, x, freqs, w, positions=p, interleaved=inter)[1]
        u = 2.0 ** -8 if w.dtype == torch.bfloat16 else 2.0 ** -24
        assert bool(((grads[2 + i].double() - dw).abs() <= 2 * u * dw.abs() + 0.005 * dw.std()).all())
