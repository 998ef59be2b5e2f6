"""Attention over the 4-bit cache where one wave of the kernel for few rows takes more than 64 tiles of 32 keys, so
that it looks into the table again: batches that fill the chip, on long caches."""
import pytest
import torch

from oracle import layer_oracle as L
from tests.test_gpu_exact import check_forward
from tests.test_gpu_fp4_cache import DT, rows

pytestmark = pytest.mark.gpu

W = 4                                                      # waves of a workgroup, which take its tiles in turn


# dtype, B, H, H_kv, nq, page, workgroups that share a row's keys, table's room
@pytest.mark.parametrize("dt,B,H,Hkv,nq,page,splits,room", [
    ("bf16", 64, 16, 8, 8, 32, 1, 17024), ("f32", 64, 8, 8, 5, 32, 1, 17024), ("bf16", 64, 8, 8, 1, 1024, 1, 17408),
    ("bf16", 32, 32, 8, 4, 64, 2, 34048),
])
def test_waves_of_many_tiles(gpu, dt, B, H, Hkv, nq, page, splits, room):
    """Scores of some tens, so that a row goes by few keys: a page that is read for another shows. Lengths end before, at and
    behind the 64th and 128th tile of each wave."""
    d, pool = 32, 61
    gen = torch.Generator("cuda").manual_seed(nq)
    k, v = (rows(gen, "bf16", 1, Hkv, pool * page, d, spread=False) for _ in range(2))
    cache = gpu.fp4_cache(pool, Hkv, page, d)
    gpu.fp4_cache_write(cache, k, v, torch.arange(pool, dtype=torch.int32, device="cuda")[None])
    m = room // page
    table = torch.randint(0, pool, (B, m), generator=gen, device="cuda", dtype=torch.int32)
    table[torch.rand(B, m, generator=gen, device="cuda") < 0.02] = -1
    table[:, 0] = 0
    turn = 64 * W * splits * 32                            # keys up to a wave's next look
    ends = [t * turn + 32 * w + x for t in (1, 2) for w in range(W + 1) for x in (-1, 0, 1)] + [0, 1, 31, room, room - 1]
    ends = [e for e in ends if e <= room]
    lengths = torch.tensor([ends[i % len(ends)] for i in range(B)], dtype=torch.int32, device="cuda")
    q = 3 * rows(gen, dt, B, H, nq, d, spread=False)
    lse = torch.empty(B, H, nq, device="cuda")
    z = gpu.fp4_cache_attention(q, cache, table, lengths, scale=1.0, lse_out=lse)
    need = gpu.fp4_attention_workspace_bytes(q, cache, table, lengths)
    assert need == (splits * B * H * nq * (d + 2) * 4 if splits > 1 else 0)
    assert torch.equal(gpu.fp4_cache_attention(q, cache, table, lengths, scale=1.0), z)
    held = [L.held(x)[0][0] for x in (k, v)]
    tokens = torch.arange(room, device="cuda")
    for b in range(B):
        page_of = table[b].long()[tokens // page]
        at = page_of.clamp(min=0) * page + tokens % page
        K, V = (x[:, at][None] for x in held)
        o = dict(scale=1.0, lengths=lengths[b:b + 1], key_mask=(page_of >= 0)[None])
        check_forward(z[b:b + 1], lse[b:b + 1], q[b:b + 1], K, V, o)
