"""Sizes that exact attention's launches do not take are refused before anything is enqueued."""
import ctypes

import pytest

from paper_2207_10284_amd import ops

INVALID, UNSUPPORTED = 1, 2
A = 1 << 20            # a fake, 16-byte aligned address: never dereferenced


def statuses(**sizes):
    """Status of forward and backward with a tensor missing: a size is refused before it is looked for."""
    p = ops._Problem(1, 2, 1, 40, 70, 32, 1, 0.125, 0, None, None, None, 0, None, 0, 0, None, 0)
    for n, x in sizes.items():
        setattr(p, n, x)
    lib, r = ops.load_exact(), ctypes.byref
    t, none = r(ops._Strided(A, 0, 0, 32)), r(ops._Strided(None, 0, 0, 0))
    fwd = lib.mra_exact_forward(r(p), none, t, t, t, None, A, 1 << 60, None)
    bwd = lib.mra_exact_backward(r(p), none, none, t, t, t, A, t, t, t, A if p.bias else None, A, 1 << 60, None)
    room = lib.mra_exact_backward_workspace_bytes(r(p))
    return fwd, bwd, room > 0


# below 2^32 threads of a launch dimension, 256 a workgroup: at most 2^24 - 1 workgroups
@pytest.mark.parametrize("sizes,forward,backward", [
    (dict(B=1 << 24, H=2, H_kv=2, n_q=1, n_k=1), UNSUPPORTED, UNSUPPORTED),
    (dict(B=1 << 24, H=1, H_kv=1, n_q=1, n_k=1), UNSUPPORTED, UNSUPPORTED),
    (dict(B=(1 << 24) - 1, H=1, H_kv=1, n_q=1, n_k=1), INVALID, INVALID),
    (dict(B=1 << 23, H=1, H_kv=1, n_q=32, n_k=1), INVALID, INVALID),
    (dict(B=1 << 23, H=1, H_kv=1, n_q=40, n_k=1), UNSUPPORTED, INVALID),             # 40 rows: two workgroups
    (dict(B=1 << 23, H=1, H_kv=1, n_q=129, n_k=1), UNSUPPORTED, UNSUPPORTED),
    (dict(B=1 << 12, H=64, H_kv=1, n_q=1, n_k=1 << 13), INVALID, INVALID),           # 2^18 workgroups each
    (dict(B=1 << 12, H=64, H_kv=64, n_q=1, n_k=1 << 13), INVALID, UNSUPPORTED),      # dK, dV: 2^24
    (dict(B=1 << 12, H=64, H_kv=64, n_q=1, n_k=(1 << 13) - 128), INVALID, INVALID),
    (dict(B=1, H=1 << 24, H_kv=1 << 24, n_q=0, n_k=1, bias=A, buckets=8, bucket_map=A), 0, UNSUPPORTED),
])
def test_launches_that_do_not_fit(sizes, forward, backward):
    fwd, bwd, room = statuses(**sizes)
    assert (fwd, bwd) == (forward, backward)
    assert room == (backward == INVALID)


def test_few_rows_on_many_long_caches_are_taken():
    """The keys' length bounds no launch of a forward: 256 key heads x 2^20 keys, 8 query heads to each."""
    p = ops._Problem(32, 64, 8, 1, 1 << 20, 128, 1, 0.125, 0, None, None, None, 0, None, 0, 0, None, 0)
    assert ops.load_exact().mra_exact_forward_workspace_bytes(ctypes.byref(p)) > 0
