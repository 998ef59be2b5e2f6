"""What a call writes into a tensor of the caller's is a change that autograd sees: a graph that kept the
old values refuses its backward, and a result that takes part in a graph itself is refused."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def leaf(*shape, dtype=torch.float32):
    gen = torch.Generator("cuda").manual_seed(sum(shape))
    return torch.randn(shape, generator=gen, device="cuda").to(dtype).requires_grad_(True)


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("which", ["q", "k"])
def test_rows_kept_for_the_backward_of_rotary(gpu, path, which):
    x, w = leaf(1, 2, 9, 32), leaf(32)
    freqs = gpu.rotary_frequencies(32)
    q, k = x * 1.0, x * 2.0
    if path == "native":
        y = gpu.rotary(q, k, freqs, q_weight=w, k_weight=w)
    else:
        y = gpu.Rotary.apply(q, k, w, w, freqs, None, False, 1.0, 1e-6)
    y[0].sum().backward(retain_graph=True)
    with torch.no_grad():
        if which == "q":
            gpu.rotary_forward(q, None, freqs, q_out=q)
        else:
            gpu.rotary_forward(q, k, freqs, k_out=k)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        (y[0].sum() + y[1].sum()).backward()


def test_a_producer_that_kept_its_result(gpu):
    x = leaf(1, 2, 9, 32)
    q = x.exp()
    with torch.no_grad():
        gpu.rotary_forward(q, None, gpu.rotary_frequencies(32), q_out=q)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        q.sum().backward()


def test_versions_go_up(gpu):
    q, k = leaf(2, 4, 9, 64).detach(), leaf(2, 2, 9, 64).detach()
    freqs = gpu.rotary_frequencies(64)
    cache = gpu.fp4_cache(4, 2, 32, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lengths = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    a, b, lse = torch.empty_like(q), torch.empty_like(k), torch.empty(2, 4, 9, device="cuda")
    calls = (
        (lambda: gpu.rotary_forward(q, k, freqs, q_out=a, k_out=b), (a, b), (q, k, freqs)),
        (lambda: gpu.rotary_forward(q, k, freqs, k_out=b), (b,), (q, k, a)),
        (lambda: gpu.rotary_backward(q, k, freqs=freqs, dq=a, dk=b), (a, b), (q, k, freqs)),
        (lambda: gpu.fp4_cache_write(cache, k, k, table), (cache.data,), (k, table)),
        (lambda: gpu.fp4_cache_read(cache, table, 9, dtype=torch.float32, k_out=a[:, :2], v_out=b), (a, b), (table, cache.data)),
        (lambda: gpu.fp4_cache_attention(q, cache, table, lengths, out=a, lse_out=lse), (a, lse), (q, cache.data, lengths)),
    )
    for call, written, read in calls:
        before = [t._version for t in (*written, *read)]
        call()
        now = [t._version for t in (*written, *read)]
        n = len(written)
        assert all(x > y for x, y in zip(now[:n], before[:n])) and now[n:] == before[n:]
    # a refused call has written nothing
    before = a._version
    with pytest.raises(gpu.MraError):
        gpu.rotary_forward(q, None, freqs, magnitude=float("inf"), q_out=a)
    assert a._version == before


def test_results_that_take_part_in_a_graph_are_refused(gpu):
    x, k = leaf(2, 4, 9, 64), leaf(2, 2, 9, 64).detach()
    q, y = x.detach(), x * 1.0
    freqs = gpu.rotary_frequencies(64)
    cache = gpu.fp4_cache(4, 2, 32, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    lengths = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    lse = torch.empty(2, 4, 9, device="cuda", requires_grad=True)
    rows = torch.empty(2, 2, 9, 64, device="cuda", requires_grad=True)
    for t in (x, y):
        for name, call in (
                ("q_out", lambda: gpu.rotary_forward(t, k, freqs, q_out=t)),
                ("q_out", lambda: gpu.rotary_forward(q, k, freqs, q_out=t)),
                ("k_out", lambda: gpu.rotary_forward(k, q, freqs, k_out=t)),
                ("dq", lambda: gpu.rotary_backward(q, k, freqs=freqs, dq=t)),
                ("dk", lambda: gpu.rotary_backward(k, q, freqs=freqs, dk=t)),
                ("out", lambda: gpu.fp4_cache_attention(q, cache, table, lengths, out=t)),
                ("lse_out", lambda: gpu.fp4_cache_attention(q, cache, table, lengths, lse_out=lse)),
                ("k_out", lambda: gpu.fp4_cache_read(cache, table, 9, dtype=torch.float32, k_out=rows)),
                ("v_out", lambda: gpu.fp4_cache_read(cache, table, 9, dtype=torch.float32, v_out=rows))):
            before = [s._version for s in (x, y, lse, rows)]
            with pytest.raises(ValueError, match=f"{name} must not require a gradient"):
                call()
            assert [s._version for s in (x, y, lse, rows)] == before
            with torch.no_grad():                          # as torch's own in-place calls
                call()


def test_inference_tensors(gpu):
    """They have no version; results allocated in inference mode are written in and out of it."""
    freqs = gpu.rotary_frequencies(32)
    with torch.inference_mode():
        q = torch.ones(1, 2, 9, 32, device="cuda")
        want = gpu.rotary_forward(q, None, freqs)[0]
        gpu.rotary_forward(q, None, freqs, q_out=q)
    assert torch.equal(q, want)
    gpu.rotary_forward(q, None, freqs, q_out=q)
