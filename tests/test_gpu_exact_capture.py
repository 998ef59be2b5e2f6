"""A captured backward of leaves of which an eager graph is alive is refused. The refusal alone is
called here, inside captures of forward calls: no such backward is run."""
import pytest
import torch

from tests.test_gpu_exact import pieces

pytestmark = pytest.mark.gpu


def captured(call):
    """call() inside a capture, on torch's capturing stream: its result, and the text of what it raised (the
    exception itself would keep the graph alive)."""
    graph, result, error = torch.cuda.CUDAGraph(), None, None
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        try:
            result = call()
        except RuntimeError as e:
            error = str(e)
    return result, error


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("which", ["q", "bias"])
def test_eager_graph_alive(gpu, path, which):
    q, k, v, _, o = pieces(gpu, "bf16", mask="l", buckets=(8, 20, True))
    bias = o.pop("bias")
    tensors = dict(q=q, k=k, v=v, bias=bias)
    tensors[which] = tensors[which].clone().requires_grad_(True)
    leaf = tensors[which]

    def forward():
        t = [tensors[n] for n in ("q", "k", "v", "bias")]
        if path == "native":
            return gpu.exact_attention(*t[:3], bias=t[3], **o)
        return gpu.ExactAttention.apply(*t, o["buckets"], o["lengths"], None, None, None, False)

    def both():
        z = forward()
        gpu.bind_exact().check_capture(z)
        return z

    z, error = captured(both)                      # no other graph
    assert error is None and z.requires_grad
    del z
    eager = leaf * 2.0                             # alive, made on the default stream
    z, error = captured(both)
    assert error is not None and "eager graph" in error
    del z
    gpu.bind_exact().check_capture(forward())      # not captured: nothing to refuse
    del eager
    side = torch.cuda.Stream()                     # a graph of another stream can be waited for
    with torch.cuda.stream(side):
        eager = leaf * 2.0
    z, error = captured(both)
    assert error is None
    del z, eager
    z, error = captured(both)
    assert error is None
