"""Second derivatives of exact attention, which it does not have: they raise, and
where autograd cannot see that one is asked for, a warning says so."""
import warnings

import pytest
import torch

from tests.test_gpu_exact import pieces, same

pytestmark = pytest.mark.gpu


def leaves_and_call(gpu, path, dt="bf16"):
    q, k, v, g, o = pieces(gpu, dt, mask="l", causal=True, buckets=(8, 20, True))
    bias = o.pop("bias")
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v, bias)]
    if path == "native":
        return leaves, lambda: gpu.exact_attention(*leaves[:3], bias=leaves[3], **o)
    return leaves, lambda: gpu.ExactAttention.apply(*leaves, o["buckets"], o["lengths"], None, None, None, True)


@pytest.mark.parametrize("path", ["native", "python"])
def test_penalty_on_the_gradient_raises(gpu, path):
    """Alone and added to another loss; the gradients themselves are what they are without a graph."""
    leaves, call = leaves_and_call(gpu, path)
    loss = call().float().square().sum()
    plain = torch.autograd.grad(loss, leaves, retain_graph=True)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        first = torch.autograd.grad(loss, leaves, create_graph=True)
    same(first, plain)
    assert all(t.requires_grad for t in first)
    for total in (first[0].float().square().sum(), loss + first[1].float().square().sum(), loss + first[3].float().sum()):
        with pytest.raises(RuntimeError, match="differentiate twice"):
            torch.autograd.grad(total, leaves, retain_graph=True, allow_unused=True)


@pytest.mark.parametrize("path", ["native", "python"])
def test_some_leaves_only(gpu, path):
    leaves, call = leaves_and_call(gpu, path, "f32")
    leaves[3].requires_grad_(False)
    loss = call().square().sum()
    first = torch.autograd.grad(loss, leaves[:3], create_graph=True)
    with pytest.raises(RuntimeError, match="differentiate twice"):
        (loss + first[2].square().sum()).backward()


@pytest.mark.parametrize("path", ["native", "python"])
def test_a_constant_gradient_of_the_output_warns(gpu, path):
    """As for a sum: what comes back is a constant to autograd (torch asks the output's gradient alone)."""
    leaves, call = leaves_and_call(gpu, path)
    out = call()
    with pytest.warns(UserWarning, match="not differentiable"):
        first = torch.autograd.grad(out.float().sum(), leaves, create_graph=True)
    assert not any(t.requires_grad for t in first)
    out = call()
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        torch.autograd.grad(out.float().sum(), leaves)


@pytest.mark.parametrize("path", ["native", "python"])
def test_without_a_bias(gpu, path):
    q, k, v, _, _ = pieces(gpu, "bf16")
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v)]
    call = gpu.exact_attention if path == "native" else (
        lambda *t: gpu.ExactAttention.apply(*t, None, None, None, None, None, None, False))
    loss = call(*leaves).float().square().sum()
    first = torch.autograd.grad(loss, leaves[1], create_graph=True)[0]
    with pytest.raises(RuntimeError, match="differentiate twice"):
        torch.autograd.grad(loss + first.float().sum(), leaves[0], retain_graph=True)
    same(torch.autograd.grad(loss, leaves[1]), (first.detach(),))
