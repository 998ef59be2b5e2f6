"""Queries with a NaN or an infinity over the 4-bit cache: their scores are NaN, so their results are, in
every kernel, with the keys of a row in one workgroup and split over several; other rows keep their bits."""
import math

import pytest
import torch

from tests.test_gpu_fp4_cache import DT, attend

pytestmark = pytest.mark.gpu

# dtype, B, H, H_kv, nq, nk, d, page, table's room, the keys are split. Few rows a key head go to the token kernel,
# 65 and more through a table with room for 2^20 tokens, or of many heads, to the one for many rows.
CASES = [(dt, 2, 4, 2, nq, nk, d, 32, wide, split)
         for dt in ("bf16", "f32") for d in (32, 64, 128)
         for nq, nk, wide, split in ((1, 700, 0, False), (1, 700, 1 << 13, True), (9, 700, 1 << 13, True),
                                     (50, 700, 1 << 20, True))]
CASES += [("bf16", 24, 32, 16, 130, 140, 128, 64, 0, False), ("f32", 24, 32, 16, 130, 140, 64, 64, 0, False)]


@pytest.mark.parametrize("case", range(len(CASES)))
def test_non_finite_queries(gpu, case):
    dt, B, H, Hkv, nq, nk, d, page, wide, split = CASES[case]
    print("non-finite", CASES[case], flush=True)
    q, cache, table, lengths, z, lse = attend(gpu, 90 + case, dt, B, H, Hkv, nq, nk, d, page, wide=wide, ragged=False)
    assert (gpu.fp4_attention_workspace_bytes(q, cache, table, lengths) > 0) == split
    bad = torch.zeros(B, H, nq, dtype=torch.bool, device="cuda")
    x = q.clone()
    for n, value in enumerate((math.nan, math.inf, -math.inf)):
        b, h, i = n % B, n % H, n * 7 % nq
        x[b, h, i, n * 11 % d] = value
        bad[b, h, i] = True
    lse2 = torch.empty_like(lse)
    z2 = gpu.fp4_cache_attention(x, cache, table, lengths, causal=True, lse_out=lse2)
    assert bool(z2[bad].isnan().all()) and bool(lse2[bad].isnan().all())
    assert torch.equal(z2[~bad], z[~bad]) and torch.equal(lse2[~bad], lse[~bad])
    # a whole row of one of them, all rows
    for value in (math.nan, math.inf, -math.inf):
        z2 = gpu.fp4_cache_attention(torch.full_like(q, value), cache, table, lengths, causal=True, lse_out=lse2)
        assert bool(z2.isnan().all()) and bool(lse2.isnan().all())


@pytest.mark.parametrize("dt", list(DT))
@pytest.mark.parametrize("nq,wide", [(1, 0), (1, 1 << 13), (50, 1 << 20)])
def test_without_a_key_they_give_zeros(gpu, dt, nq, wide):
    """No score, so nothing that could be NaN: empty sequences, positions before the first token, no pages."""
    q, cache, table, lengths, _, lse = attend(gpu, 7, dt, 2, 4, 2, nq, 700, 64, 32, wide=wide, ragged=False)
    x = torch.full_like(q, math.nan)
    far = torch.full_like(lengths, -nq)
    for kw in (dict(lengths=0 * lengths), dict(q_start=far), dict(table=torch.full_like(table, -1))):
        a = dict(table=table, lengths=lengths, q_start=None)
        a.update(kw)
        z = gpu.fp4_cache_attention(x, cache, a["table"], a["lengths"], causal=True, q_start=a["q_start"], lse_out=lse)
        assert not z.any() and bool((lse == -math.inf).all())
