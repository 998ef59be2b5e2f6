"""Sizes at the border of a launch of libmra_layer: one that fits is not refused for its size (here for a missing tensor, before
anything is enqueued), the next one is."""
import pytest

from paper_2207_10284_amd import ops
from tests.test_layer_cpu import INVALID, UNSUPPORTED, cache, rows, tensor


# a workgroup takes 64 neighbouring tokens of one head, aligned; below 2^24 workgroups
@pytest.mark.parametrize("n", [1, 2, 33, 64, 65, 66, 130, 1 << 10, 100001, 1 << 20, 1 << 26])
@pytest.mark.parametrize("read", [False, True])
def test_cache_calls_of_every_size_that_fits(n, read):
    lib = ops.load_layer()
    tiles = max((63 + n - 1) // 64 + 1, 1)                 # the first token at the end of a tile
    most = ((1 << 24) - 1) // tiles
    for H in (1, 2, 8):
        if most >= H:
            assert rows(lib, cache(B=most // H, H_kv=H), n=n, read=read, k=tensor(None)) == INVALID
        assert rows(lib, cache(B=most // H + 1, H_kv=H), n=n, read=read, k=tensor(None)) == UNSUPPORTED


@pytest.mark.parametrize("size,d", [((1 << 32) + 32, 64), (32 - (1 << 32), 64), (32, (1 << 32) + 64), (1 << 70, 64), (-32, 64)])
def test_pages_of_sizes_past_32_bits(size, d):
    assert ops.fp4_page_bytes(size, d) == 0
    with pytest.raises(ValueError, match="page_size"):
        ops.fp4_cache(2, 2, size, d, device="cpu")
