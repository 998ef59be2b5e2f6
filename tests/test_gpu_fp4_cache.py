"""The 4-bit cache on the GPU: what is written, what comes back, and attention over it.

Written values are compared bit for bit with the float64 oracle (every step of the
definition is exact). Attention is held to the bounds of tests/test_gpu_exact.py on the
held values, which are exact in both types."""
import math

import pytest
import torch

from oracle import layer_oracle as L
from tests.test_gpu_exact import check_forward

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def rows(gen, dt, B, h, n, d, layout="bhnd", spread=True):
    x = torch.randn((B, n, h, d) if layout == "bnhd" else (B, h, n, d), generator=gen, device="cuda")
    if spread:
        x = x * torch.exp(2 * torch.randn(x.shape[:-1] + (d // 32, 1), generator=gen, device="cuda")).expand(
            *x.shape[:-1], d // 32, 32).reshape(x.shape)
    x = x.to(DT[dt])
    return x.transpose(1, 2) if layout == "bnhd" else x


def table_of(gen, B, m, pages):
    return torch.randperm(pages, generator=gen, device="cuda")[: B * m].view(B, m).to(torch.int32)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def live(counts, n):
    return (torch.arange(n, device="cuda") < counts[:, None])[:, None, :, None]


# dtype, B, H_kv, n, d, page size, pages of a sequence, layout, starts, counts
WRITES = [
    ("bf16", 1, 1, 1, 64, 32, 1, "bhnd", None, None),
    ("f32", 2, 3, 33, 32, 32, 3, "bnhd", (5, 31), (33, 20)),
    ("bf16", 3, 2, 100, 128, 64, 4, "bnhd", (0, 63, 130), (100, 0, 77)),
    ("f32", 2, 2, 257, 128, 128, 3, "bhnd", (1, 127), None),
    ("bf16", 2, 5, 64, 64, 32, 2, "bhnd", None, (64, 40)),
    ("bf16", 33, 4, 1, 64, 64, 3, "bnhd", tuple(range(0, 165, 5)), None),
    ("bf16", 2, 1, 7, 32, 1024, 1, "bhnd", (6, 1020), None),                          # the second runs past its page
    ("f32", 2, 2, 2, 64, 32, 2, "bhnd", (31, 7), None),                               # across two pages
    ("bf16", 1, 2, 0, 64, 32, 2, "bhnd", None, None),
]


@pytest.mark.parametrize("case", range(len(WRITES)))
def test_written_and_read_back(gpu, case):
    dt, B, H, n, d, page, m, layout, starts, counts = WRITES[case]
    print("cache", WRITES[case], flush=True)
    gen = torch.Generator("cuda").manual_seed(case)
    k, v = rows(gen, dt, B, H, n, d, layout), rows(gen, dt, B, H, n, d, layout)
    cache = gpu.fp4_cache(B * m + 2, H, page, d)
    cache.data.random_(0, 256, generator=gen)
    before = cache.data.clone()
    table = table_of(gen, B, m, B * m + 2)
    s = None if starts is None else ints(*starts)
    c = None if counts is None else ints(*counts)
    gpu.fp4_cache_write(cache, k, v, table, starts=s, counts=c)
    s0 = torch.zeros(B, dtype=torch.int32, device="cuda") if s is None else s
    c0 = torch.full((B,), n, dtype=torch.int32, device="cuda") if c is None else c
    c0 = torch.minimum(c0, m * page - s0)
    for out in ("bf16", "f32"):
        kr, vr = gpu.fp4_cache_read(cache, table, n, starts=s, counts=c, dtype=DT[out])
        for got, x in ((kr, k), (vr, v)):
            want = torch.where(live(c0, n), L.held(x)[0], 0.0)
            assert torch.equal(got.double(), want)
    # only the bytes of these tokens have changed
    used = torch.zeros(B * m + 2, page, dtype=torch.bool, device="cuda")
    for b in range(B):
        t = torch.arange(int(c0[b]), device="cuda") + int(s0[b])
        used[table[b].long()[t // page], t % page] = True
    parts = [used[:, :, None].expand(-1, -1, x).reshape(len(used), -1) for x in (d // 2, d // 2, d // 32, d // 32)]
    mask = torch.cat(parts, 1)[:, None].expand_as(before)
    assert mask.shape[2] == cache.data.shape[2]
    assert torch.equal(cache.data[~mask], before[~mask])


@pytest.mark.parametrize("d", [32, 64, 128])
def test_the_bytes_are_the_layouts(gpu, d):
    gen = torch.Generator("cuda").manual_seed(d)
    k, v = rows(gen, "bf16", 1, 2, 64, d), rows(gen, "bf16", 1, 2, 64, d)
    cache = gpu.fp4_cache(3, 2, 64, d)
    gpu.fp4_cache_write(cache, k, v, ints(2)[None])
    for h in range(2):
        want = L.page_bytes(k[0, h].cpu(), v[0, h].cpu())
        got = cache.data[2, h].cpu()
        # a zero may carry a sign: codes 8 and 0
        codes = 64 * d
        g, w = got[:codes], want[:codes]
        for shift in (0, 4):
            a, b = g >> shift & 15, w >> shift & 15
            assert torch.equal(torch.where(a == 8, 0, a), torch.where(b == 8, 0, b))
        assert torch.equal(got[codes:], want[codes:])
    assert not cache.data[:2].any()


def test_every_border_and_tie(gpu):
    """All borders between codes, their neighbours in both types, at steps over the whole range."""
    grid = torch.tensor(L.GRID, dtype=torch.float64)
    mid = (grid[1:] + grid[:-1]) / 2
    for dt, ulp in (("f32", 2.0 ** -23), ("bf16", 2.0 ** -7)):
        x = torch.cat([grid, mid, mid * (1 + ulp), mid * (1 - ulp), torch.tensor([6.5, 7.0, 7.0 * (1 - ulp), 6.0 * (1 - ulp)])])
        x = torch.cat([x, -x]).to(DT[dt]).double()
        x = torch.cat([x, torch.zeros(-len(x) % 30)])
        blocks = torch.cat([x.view(-1, 30), torch.full((len(x) // 30, 1), 7.0), torch.full((len(x) // 30, 1), -4.0)], 1)
        tops = torch.stack([torch.full((32,), t) for t in (7.0, 7.0 * (1 + ulp), 3.5, 3.5 * (1 + ulp), 4.0, 5.25, 0.0)])
        blocks = torch.cat([blocks, tops.double()])
        scales = torch.tensor([2.0 ** e for e in (-125, -124, -120, -60, -1, 0, 1, 50, 120, 124, 125)], dtype=torch.float64)
        scales = scales[scales * 8 < torch.finfo(DT[dt]).max]
        rows_ = (blocks[None] * scales[:, None, None]).reshape(-1, 32).to(DT[dt]).cuda()
        extra = torch.full((2, 32), torch.finfo(DT[dt]).max, dtype=DT[dt], device="cuda")
        extra[1] = torch.finfo(DT[dt]).tiny
        rows_ = torch.cat([rows_, extra])
        n = len(rows_)
        k = rows_.view(1, 1, n, 32)
        cache = gpu.fp4_cache(n // 32 + 1, 1, 32, 32)
        table = torch.arange(n // 32 + 1, dtype=torch.int32, device="cuda")[None]
        gpu.fp4_cache_write(cache, k, -k, table)
        kr, vr = gpu.fp4_cache_read(cache, table, n, dtype=torch.float32)
        want = L.held(k)[0]
        assert torch.equal(kr.double(), want) and torch.equal(vr.double(), -want)
        assert kr.isfinite().all() and torch.equal(kr.bfloat16().float(), kr)


def test_infinities_and_nan(gpu):
    """An infinity is the largest held value, its block's steps 2^125; a NaN's block is finite."""
    k = torch.randn(1, 1, 32, 64, device="cuda")
    k[0, 0, 3, 5], k[0, 0, 4, 40], k[0, 0, 5, 0] = math.inf, -math.inf, math.nan
    cache = gpu.fp4_cache(1, 1, 32, 64)
    gpu.fp4_cache_write(cache, k, k, ints(0)[None])
    kr, vr = gpu.fp4_cache_read(cache, ints(0)[None], 32, dtype=torch.float32)
    top = 6 * 2.0 ** 125
    assert kr[0, 0, 3, 5] == top and kr[0, 0, 4, 40] == -top and kr.isfinite().all() and torch.equal(kr, vr)
    keep = torch.ones(32, 2, dtype=torch.bool, device="cuda")
    keep[3, 0] = keep[4, 1] = keep[5, 0] = False
    keep = keep.repeat_interleave(32, 1)
    assert torch.equal(kr[0, 0].double()[keep], L.held(torch.nan_to_num(k, 0.0, 0.0, 0.0))[0][0, 0][keep])


def test_bad_pages(gpu):
    """Entries outside the cache are no pages: not written, read as zeros, not attended to."""
    gen = torch.Generator("cuda").manual_seed(4)
    B, H, d, page, m = 2, 2, 64, 32, 4
    k, v = rows(gen, "bf16", B, H, m * page, d), rows(gen, "bf16", B, H, m * page, d)
    table = table_of(gen, B, m, B * m)
    bad = table.clone()
    bad[0, 1], bad[1, 0], bad[1, 3] = -1, B * m, 2 ** 31 - 1
    cache = gpu.fp4_cache(B * m, H, page, d)
    gpu.fp4_cache_write(cache, k, v, bad)
    for i, j in ((0, 1), (1, 0), (1, 3)):
        assert not cache.data[table[i, j].item()].any()
    ok = (bad == table).repeat_interleave(page, 1)
    kr, vr = gpu.fp4_cache_read(cache, bad, m * page)
    for got, x in ((kr, k), (vr, v)):
        assert torch.equal(got.double(), torch.where(ok[:, None, :, None], L.held(x)[0], 0.0))
    for nq, wide in ((1, 0), (5, 0), (70, 0), (70, 1 << 20)):
        if wide:
            bad = torch.cat([bad, torch.full((B, wide // page), -1, dtype=torch.int32, device="cuda")], 1)
        q = rows(gen, "bf16", B, 4, nq, d, spread=False)
        lengths = ints(m * page, m * page - 3)
        lse = torch.empty(B, 4, nq, device="cuda")
        z = gpu.fp4_cache_attention(q, cache, bad, lengths, causal=True, lse_out=lse)
        check_forward(z, lse, q, kr, vr, dict(scale=None, causal=True, lengths=lengths, key_mask=ok,
                                              q_start=lengths - nq))


def attend(gpu, seed, dt, B, H, Hkv, nq, nk, d, page, layout="bhnd", causal=True, ragged=True, start=None, scale=None,
           kv="bf16", empty=False, wide=0):
    gen = torch.Generator("cuda").manual_seed(seed)
    k, v = rows(gen, kv, B, Hkv, nk, d, spread=False), rows(gen, kv, B, Hkv, nk, d, spread=False)
    q = rows(gen, dt, B, H, nq, d, layout, spread=False)
    m = -(-nk // page)
    cache = gpu.fp4_cache(B * m + 1, Hkv, page, d)
    cache.data.fill_(255)                                  # behind the sequences lies anything
    table = table_of(gen, B, m, B * m + 1)
    if wide:                                               # entries that no length reaches
        table = torch.cat([table, torch.full((B, wide // page - m), -1, dtype=torch.int32, device="cuda")], 1)
    lengths = torch.full((B,), nk, dtype=torch.int32, device="cuda")
    if ragged:
        lengths = torch.randint(0, nk + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    if empty and B:
        lengths[0] = 0
    gpu.fp4_cache_write(cache, k, v, table, counts=lengths)
    s = None if start is None else torch.randint(*start, (B,), generator=gen, device="cuda", dtype=torch.int32)
    lse = torch.empty(B, H, nq, device="cuda")
    z = gpu.fp4_cache_attention(q, cache, table, lengths, scale=scale, causal=causal, q_start=s, lse_out=lse)
    torch.cuda.synchronize()
    o = dict(scale=scale, causal=causal, lengths=lengths, q_start=lengths - nq if s is None else s)
    check_forward(z, lse, q, L.held(k)[0], L.held(v)[0], o)
    return q, cache, table, lengths, z, lse


# dtype, B, H, H_kv, nq, nk, d, page size, options
ATTENDS = [
    ("bf16", 1, 1, 1, 1, 1, 64, 32, dict(ragged=False)),
    ("f32", 1, 1, 1, 1, 1, 32, 32, dict(ragged=False)),
    ("bf16", 3, 12, 12, 1, 300, 64, 32, {}),
    ("bf16", 2, 16, 4, 1, 1000, 128, 64, {}),
    ("f32", 2, 4, 2, 1, 700, 128, 256, {}),
    ("bf16", 4, 8, 1, 1, 513, 32, 128, dict(empty=True)),
    ("f32", 3, 6, 3, 2, 129, 64, 32, {}),
    ("bf16", 2, 8, 2, 5, 260, 64, 64, dict(layout="bnhd")),
    ("bf16", 2, 32, 1, 3, 100, 128, 32, {}),
    ("bf16", 1, 16, 16, 33, 90, 32, 32, dict(causal=False)),
    ("f32", 2, 8, 2, 40, 333, 32, 64, dict(layout="bnhd")),
    ("bf16", 2, 4, 2, 150, 150, 64, 32, dict(ragged=False)),
    ("bf16", 2, 4, 1, 200, 900, 128, 128, {}),
    ("f32", 1, 4, 4, 257, 300, 64, 32, {}),
    ("f32", 1, 2, 1, 129, 500, 128, 32, dict(causal=False)),
    ("bf16", 2, 2, 2, 100, 64, 64, 64, dict(ragged=False)),                           # the first rows have no key
    ("bf16", 2, 4, 2, 7, 200, 64, 32, dict(start=(-40, 240))),
    ("f32", 2, 4, 2, 70, 200, 128, 32, dict(start=(-100, 300))),
    ("bf16", 2, 4, 2, 1, 4000, 64, 64, dict(scale=1.0, ragged=False)),
    ("bf16", 2, 4, 2, 1, 2000, 128, 1024, dict(scale=0.01)),
    ("bf16", 64, 16, 8, 33, 161, 64, 32, {}),
    ("bf16", 2, 4, 2, 0, 64, 64, 32, {}),
    ("bf16", 0, 4, 2, 3, 64, 64, 32, {}),
    ("f32", 2, 4, 2, 3, 0, 64, 32, dict(ragged=False)),
    ("bf16", 1, 64, 1, 1, 5000, 128, 64, dict(kv="f32")),
    ("bf16", 1, 8, 8, 1, 20000, 32, 32, dict(kv="f32")),
    ("f32", 1, 40, 8, 1, 9000, 64, 512, dict(kv="f32")),
    ("bf16", 1, 2, 2, 600, 1100, 128, 64, {}),
    ("bf16", 16, 32, 8, 90, 200, 32, 32, {}),
    ("bf16", 40, 32, 16, 70, 130, 64, 32, {}),
    ("f32", 40, 16, 16, 70, 130, 64, 32, dict(empty=True)),
    ("bf16", 24, 32, 16, 130, 140, 128, 64, dict(layout="bnhd")),
    ("f32", 40, 16, 16, 66, 100, 128, 32, dict(start=(-30, 90))),
    ("f32", 40, 32, 16, 65, 70, 32, 32, dict(causal=False)),
]


# a table with room for 2^20 tokens: more workgroups share the keys, and from 65 rows a key head on the kernel
# for many rows runs
@pytest.mark.parametrize("wide", [0, 1 << 20])
@pytest.mark.parametrize("case", range(len(ATTENDS)))
def test_attention(gpu, case, wide):
    dt, B, H, Hkv, nq, nk, d, page, opts = ATTENDS[case]
    print("attend", ATTENDS[case], wide, flush=True)
    attend(gpu, 50 + case, dt, B, H, Hkv, nq, nk, d, page, wide=wide, **opts)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("nq,wide", [(1, 0), (40, 0), (140, 1 << 20)])
@pytest.mark.parametrize("d", [64, 128])
def test_logits_of_hundreds(gpu, dt, nq, wide, d):
    """Rising and falling runs of large logits: the reference has to move."""
    gen = torch.Generator("cuda").manual_seed(7)
    n = 1500
    q = torch.zeros(1, 2, nq, d, device="cuda")
    q[..., 0] = 8.0
    q[:, 1, :, 0] = -8.0
    k = 0.01 * torch.randn(1, 2, n, d, generator=gen, device="cuda")
    k[..., 0] = torch.linspace(-500, 500, n, device="cuda")
    v = torch.randn(1, 2, n, d, generator=gen, device="cuda")
    cache = gpu.fp4_cache(n // 32 + 1, 2, 32, d)
    table = torch.full((1, max(n, wide) // 32 + 1), -1, dtype=torch.int32, device="cuda")
    table[0, : n // 32 + 1] = torch.arange(n // 32 + 1)
    gpu.fp4_cache_write(cache, k, v, table)
    lse = torch.empty(1, 2, nq, device="cuda")
    q = q.to(DT[dt])
    z = gpu.fp4_cache_attention(q, cache, table, ints(n), lse_out=lse)
    check_forward(z, lse, q, L.held(k)[0], L.held(v)[0], dict(scale=None, lengths=ints(n)))


def test_lengths_beyond_the_table_are_its_end(gpu):
    q, cache, table, lengths, _, _ = attend(gpu, 3, "bf16", 2, 4, 2, 3, 128, 64, 32, ragged=False)
    z = gpu.fp4_cache_attention(q, cache, table, lengths, causal=True)
    far = gpu.fp4_cache_attention(q, cache, table, lengths + 1000, causal=True)
    assert torch.equal(z, far)
    none = gpu.fp4_cache_attention(q, cache, table, lengths * 0 - 5, causal=True)
    assert not none.any()


def test_results_do_not_depend_on_where_the_pages_lie(gpu):
    gen = torch.Generator("cuda").manual_seed(13)
    for nq, wide in ((1, 0), (60, 0), (60, 1 << 20)):
        q, cache, table, lengths, z, _ = attend(gpu, 14, "bf16", 3, 8, 2, nq, 700, 64, 32, wide=wide)
        order = torch.randperm(cache.data.shape[0], generator=gen, device="cuda")
        moved = gpu.Fp4Cache(cache.data[order].contiguous(), 32, 64)
        there = torch.where(table < 0, -1, torch.argsort(order)[table.long().clamp(min=0)]).to(torch.int32)
        assert torch.equal(gpu.fp4_cache_attention(q, moved, there, lengths, causal=True), z)


def test_shared_pages_and_wider_tables(gpu):
    """Two sequences on the same pages give the same bits; entries behind the lengths are not looked at."""
    q, cache, table, lengths, z, _ = attend(gpu, 15, "bf16", 2, 8, 2, 4, 300, 64, 32, ragged=False)
    wide = torch.full((2, table.shape[1] + 5), -7, dtype=torch.int32, device="cuda")
    wide[:, : table.shape[1]] = table[:1]
    same = gpu.fp4_cache_attention(q[:1].expand_as(q), cache, wide, lengths, causal=True)
    assert torch.equal(same[0], same[1])
    assert (same[0].float() - z[0].float()).abs().max() <= 3 * 2.0 ** -8 * z.abs().max()


def test_streams_and_workspace(gpu):
    q, cache, table, lengths, z, lse = attend(gpu, 16, "bf16", 2, 8, 2, 1, 3000, 64, 64)
    need = gpu.fp4_attention_workspace_bytes(q, cache, table, lengths)
    ws = torch.empty(need + 64, dtype=torch.uint8, device="cuda")
    assert torch.equal(gpu.fp4_cache_attention(q, cache, table, lengths, causal=True, workspace=ws), z)
    if need:
        with pytest.raises(gpu.MraError, match="WORKSPACE"):
            gpu.fp4_cache_attention(q, cache, table, lengths, causal=True, workspace=ws[: need - 16])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = gpu.fp4_cache_attention(q, cache, table, lengths, causal=True)
    side.synchronize()
    assert torch.equal(got, z)


def test_two_streams_at_once(gpu):
    """Calls on two streams, each with its own cache, share nothing."""
    a = attend(gpu, 30, "bf16", 2, 8, 2, 1, 3000, 64, 64)
    b = attend(gpu, 31, "f32", 2, 8, 2, 90, 1500, 128, 32, wide=1 << 20)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (stream, (q, cache, table, lengths, _, _)) in enumerate(zip(streams, (a, b))):
            with torch.cuda.stream(stream):
                got[i].append(gpu.fp4_cache_attention(q, cache, table, lengths, causal=True))
    torch.cuda.synchronize()
    for z, want in zip(got, (a, b)):
        assert all(torch.equal(x, want[4]) for x in z)


def test_refusals(gpu):
    q, cache, table, lengths, _, _ = attend(gpu, 32, "bf16", 2, 8, 2, 3, 100, 64, 32)
    k = torch.zeros(2, 2, 5, 64, device="cuda", dtype=torch.bfloat16)
    wide = torch.zeros(2, 2, 5, 66, device="cuda", dtype=torch.bfloat16)[..., :64]
    for bad, match in ((dict(k=k[:1]), "share shape"), (dict(v=k[:, :1]), "share shape"), (dict(v=k.float()), "v must be"),
                       (dict(k=wide), "dense rows"), (dict(table=table[:1]), "share shape"),
                       (dict(table=table.long()), "int32"), (dict(table=table[0]), "int32"),
                       (dict(starts=lengths[:1]), "starts"), (dict(counts=lengths.long()), "counts"),
                       (dict(table=table.cpu()), "int32")):
        a = dict(k=k, v=k, table=table)
        extra = {n: bad.pop(n) for n in ("starts", "counts") if n in bad}
        a.update(bad)
        with pytest.raises(ValueError, match=match):
            gpu.fp4_cache_write(cache, a["k"], a["v"], a["table"], **extra)
    with pytest.raises(TypeError, match="float16"):
        gpu.fp4_cache_write(cache, k.half(), k.half(), table)
    with pytest.raises(TypeError, match="Half|float16"):
        gpu.fp4_cache_read(cache, table, 4, dtype=torch.float16)
    with pytest.raises(ValueError, match="negative"):
        gpu.fp4_cache_read(cache, table, -1)
    with pytest.raises(ValueError, match="k_out"):
        gpu.fp4_cache_read(cache, table, 4, k_out=torch.empty(2, 2, 5, 64, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="broadcast"):
        gpu.fp4_cache_read(cache, table, 5, v_out=k[:1].expand(2, 2, 5, 64))
    for bad, match in ((dict(q=q[:1]), "q must have"), (dict(q=q[:, :7]), "q must have"), (dict(q=q[..., :32]), "q must have"),
                       (dict(lengths=lengths.long()), "lengths"), (dict(q_start=lengths[:1]), "q_start"),
                       (dict(out=q[:1].expand_as(q)), "broadcast"), (dict(out=q.float()), "out must be"),
                       (dict(lse_out=torch.empty(2, 8, 4, device="cuda")), "lse_out"),
                       (dict(workspace=torch.empty(9, 2, device="cuda")[:, 0]), "workspace")):
        a = dict(q=q, lengths=lengths)
        a.update(bad)
        with pytest.raises(ValueError, match=match):
            gpu.fp4_cache_attention(a.pop("q"), cache, table, a.pop("lengths"), **a)
    for scale in (0.0, -1.0, math.nan, math.inf):
        with pytest.raises(gpu.MraError, match="INVALID"):
            gpu.fp4_cache_attention(q, cache, table, lengths, scale=scale)


def test_a_captured_decoder_step(gpu):
    """One step of a decoder's layer as it is served: rotation of new rows, the cache written, attention; captured
    once, replayed while positions, lengths and rows change."""
    B, H, Hkv, d, page, m = 3, 8, 2, 64, 32, 6
    gen = torch.Generator("cuda").manual_seed(17)
    qkv = torch.zeros(B, 1, H + 2 * Hkv, d, device="cuda", dtype=torch.bfloat16)
    wq, wk = (1 + 0.1 * torch.randn(d, generator=gen, device="cuda") for _ in range(2))
    freqs = gpu.rotary_frequencies(d)
    table = table_of(gen, B, m, B * m)
    pos = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(B, dtype=torch.int32, device="cuda")
    caches = [gpu.fp4_cache(B * m, Hkv, page, d) for _ in range(2)]

    def step(cache):
        q, k, v = qkv.transpose(1, 2).split([H, Hkv, Hkv], 1)
        q, k = gpu.rotary_forward(q, k, freqs, positions=pos, q_weight=wq, k_weight=wk)
        gpu.fp4_cache_write(cache, k, v, table, starts=pos[:, 0])
        return gpu.fp4_cache_attention(q, cache, table, lengths, causal=True)

    step(caches[0])
    caches[0].data.zero_()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step(caches[0])
    kept = []
    for t in range(40):
        new = torch.randn(qkv.shape, generator=gen, device="cuda").to(torch.bfloat16)
        kept.append(new)
        qkv.copy_(new)
        pos.copy_(torch.tensor([[t], [t + 50], [t]]))
        lengths.copy_(pos[:, 0] + 1)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, step(caches[1])), t
    assert torch.equal(caches[0].data, caches[1].data)
    # the last step against the definition: sequences 0 and 2 hold all 40 tokens
    x = torch.cat(kept, 1).transpose(1, 2)
    q, k, v = x.split([H, Hkv, Hkv], 1)
    at = torch.arange(40, dtype=torch.int32, device="cuda")
    yq, yk = gpu.rotary_forward(q, k, freqs, positions=at, q_weight=wq, k_weight=wk)
    for b in (0, 2):
        K, V = L.held(yk[b:b + 1])[0], L.held(v[b:b + 1])[0]
        lse = torch.empty(1, H, 1, device="cuda")
        z = gpu.fp4_cache_attention(yq[b:b + 1, :, -1:], caches[1], table[b:b + 1], ints(40), lse_out=lse)
        check_forward(z, lse, yq[b:b + 1, :, -1:], K, V, dict(scale=None))
        assert torch.equal(z[0], got[b])


def test_a_prompt_and_then_tokens(gpu):
    """A prompt in pieces, then single tokens, gives what one call over everything gives."""
    B, H, Hkv, d, n = 2, 4, 2, 128, 150
    gen = torch.Generator("cuda").manual_seed(19)
    q, k, v = (rows(gen, "bf16", B, h, n, d, "bnhd", spread=False) for h in (H, Hkv, Hkv))
    cache = gpu.fp4_cache(B * 5, Hkv, 32, d)
    table = table_of(gen, B, 5, B * 5)
    whole = torch.empty(B, H, n, d, device="cuda", dtype=torch.bfloat16)
    at = 0
    for piece in (64, 60, 20, 1, 1, 1, 3):
        s = torch.full((B,), at, dtype=torch.int32, device="cuda")
        gpu.fp4_cache_write(cache, k[:, :, at:at + piece], v[:, :, at:at + piece], table, starts=s)
        gpu.fp4_cache_attention(q[:, :, at:at + piece], cache, table, s + piece, causal=True,
                                out=whole[:, :, at:at + piece])
        at += piece
    lse = torch.empty(B, H, n, device="cuda")
    z = gpu.fp4_cache_attention(q, cache, table, ints(n, n), causal=True, lse_out=lse)
    o = dict(scale=None, causal=True)
    K, V = L.held(k)[0], L.held(v)[0]
    check_forward(z, lse, q, K, V, o)
    check_forward(whole, lse, q, K, V, o)


def test_a_cache_past_32_bits(gpu):
    """Pages whose bytes begin past 2^32."""
    page, d, H = 1024, 128, 8
    per = gpu.fp4_page_bytes(page, d) * H
    pages = (5 << 30) // per
    data = torch.empty(pages, H, per // H, dtype=torch.uint8, device="cuda")
    cache = gpu.Fp4Cache(data, page, d)
    gen = torch.Generator("cuda").manual_seed(21)
    k, v = rows(gen, "bf16", 1, H, 1500, d, spread=False), rows(gen, "bf16", 1, H, 1500, d, spread=False)
    table = ints(pages - 1, pages - 2)[None]
    gpu.fp4_cache_write(cache, k, v, table)
    kr, vr = gpu.fp4_cache_read(cache, table, 1500)
    assert torch.equal(kr.double(), L.held(k)[0]) and torch.equal(vr.double(), L.held(v)[0])
    for nq, wide in ((1, 0), (50, 1 << 10)):
        if wide:
            table = torch.cat([table, table[:, :1].expand(1, wide)], 1)
        q = rows(gen, "bf16", 1, 16, nq, d, spread=False)
        lse = torch.empty(1, 16, nq, device="cuda")
        z = gpu.fp4_cache_attention(q, cache, table, ints(1500), causal=True, lse_out=lse)
        check_forward(z, lse, q, kr, vr, dict(scale=None, causal=True))


def test_cached_attention_equals_exact_attention_on_the_held_values(gpu):
    """Within the rounding of either: both are held to 3 u of the terms."""
    q, cache, table, lengths, z, _ = attend(gpu, 23, "bf16", 2, 8, 2, 40, 500, 64, 64)
    k, v = gpu.fp4_cache_read(cache, table, 500, counts=lengths)
    e = gpu.exact_attention_forward(q, k, v, causal=True, lengths=lengths, q_start=lengths - 40)
    assert (z.double() - e.double()).abs().max() <= 6 * 2.0 ** -8 * v.abs().max()
    assert math.isfinite(z.abs().max().item())
