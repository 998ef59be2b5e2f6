"""libmra_layer without a GPU: the ABI's exports and refusals, the frequencies, the
oracle's pins, and the bounds of what the kernels address in a page."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

from oracle import layer_oracle as L
from paper_2207_10284_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mra_layer.h")
OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = range(5)
A = 1 << 20            # a fake, 16-byte aligned address: never dereferenced
I, P = ctypes.c_int, ctypes.c_void_p


class Rotary(ctypes.Structure):
    _fields_ = [("B", I), ("H", I), ("H_kv", I), ("n", I), ("d", I), ("rot", I), ("dtype", I), ("interleaved", I),
                ("magnitude", ctypes.c_float), ("eps", ctypes.c_float), ("freqs", P), ("positions", P),
                ("positions_stride", ctypes.c_int64), ("q_weight", P), ("k_weight", P), ("weight_dtype", I)]


class Cache(ctypes.Structure):
    _fields_ = [("pages", I), ("H_kv", I), ("d", I), ("page_size", I), ("data", P), ("table", P), ("B", I),
                ("max_pages", I)]


class Attention(ctypes.Structure):
    _fields_ = [("H", I), ("n_q", I), ("dtype", I), ("scale", ctypes.c_float), ("causal", I), ("lengths", P),
                ("q_start", P)]


@pytest.fixture(scope="module")
def lib():
    return ops.load_layer()


def change(p, **kw):
    for n, x in kw.items():
        setattr(p, n, x)
    return p


def rotary(**kw):
    return change(Rotary(2, 4, 2, 30, 64, 64, 1, 0, 1.0, 1e-6, A, None, 0, None, None, 0), **kw)


def cache(**kw):
    return change(Cache(9, 2, 64, 32, A, A, 3, 4), **kw)


def attention(**kw):
    return change(Attention(8, 5, 1, 0.125, 1, A, None), **kw)


def tensor(data=A, b=0, h=0, n=64):
    return ctypes.byref(ops._Strided(data, b, h, n))


def turn(lib, p, **kw):
    t = [kw.get(n) or tensor() for n in ("q", "k", "q_out", "k_out")]
    return lib.mra_rotary_forward(ctypes.byref(p) if p else None, *t, None)


def turn_back(lib, p, dqw=None, dkw=None, ws=A, size=1 << 40, **kw):
    t = [kw.get(n) or tensor() for n in ("q", "k", "dq_out", "dk_out", "dq", "dk")]
    return lib.mra_rotary_backward(ctypes.byref(p) if p else None, *t, dqw, dkw, ws, size, None)


def rows(lib, c, n=7, dtype=1, read=False, k=None, v=None):
    f = lib.mra_fp4_cache_read if read else lib.mra_fp4_cache_write
    return f(ctypes.byref(c) if c else None, k or tensor(), v or tensor(), n, dtype, None, None, None)


def attend(lib, c, p, q=None, out=None, lse=None, ws=A, size=1 << 40):
    return lib.mra_fp4_attention(ctypes.byref(c) if c else None, ctypes.byref(p) if p else None, q or tensor(),
                                 out or tensor(), lse, ws, size, None)


def test_exports_are_the_header(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(mra_(?:rotary|fp4|layer)_[a-z0-9_]+)\s*\(", text))
    assert names == set(ops.LAYER_SIGNATURES)
    if shutil.which("nm"):
        out = subprocess.run(["nm", "-D", "--defined-only", ops.LAYER_LIB_PATH], capture_output=True, text=True,
                             check=True).stdout
        funcs = {line.split()[-1] for line in out.splitlines() if len(line.split()) == 3 and line.split()[1] == "T"}
        assert {f for f in funcs if not f.startswith("_Z")} == names


BAD_ROTARY = [
    (dict(B=-1), INVALID), (dict(H=-1), INVALID), (dict(H_kv=-1), INVALID), (dict(n=-1), INVALID), (dict(d=0), INVALID),
    (dict(rot=-16), INVALID), (dict(interleaved=2), INVALID), (dict(magnitude=math.nan), INVALID),
    (dict(magnitude=math.inf), INVALID), (dict(d=48, rot=32), UNSUPPORTED), (dict(rot=80), INVALID),
    (dict(rot=8), UNSUPPORTED), (dict(rot=20), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(q_weight=A, weight_dtype=7), UNSUPPORTED), (dict(q_weight=A, eps=0.0), INVALID),
    (dict(k_weight=A, eps=-1.0), INVALID), (dict(k_weight=A, eps=math.nan), INVALID), (dict(k_weight=A, eps=math.inf), INVALID),
    (dict(positions=A, positions_stride=-1), INVALID), (dict(n=(1 << 26) + 1), UNSUPPORTED),
    (dict(H=(1 << 16) + 1), UNSUPPORTED), (dict(B=1 << 17, n=1 << 10), UNSUPPORTED), (dict(freqs=None), INVALID),
]


@pytest.mark.parametrize("bad,status", BAD_ROTARY)
def test_rotary_problems_refused(lib, bad, status):
    p = rotary(**bad)
    assert turn(lib, p) == status and turn_back(lib, p) == status
    if "freqs" not in bad:
        assert lib.mra_rotary_backward_workspace_bytes(ctypes.byref(p)) == 0


BAD_TENSORS = [(tensor(None), INVALID), (tensor(A + 8), MISALIGNED), (tensor(n=-64), INVALID), (tensor(n=68), MISALIGNED),
               (tensor(n=1 << 24), UNSUPPORTED), (tensor(h=4), MISALIGNED), (tensor(b=12), MISALIGNED)]


def test_rotary_tensors_refused(lib):
    assert turn(lib, None) == INVALID and turn_back(lib, None) == INVALID
    w = rotary(q_weight=A, k_weight=A)
    for bad, status in BAD_TENSORS:
        for name in ("q", "k", "q_out", "k_out"):
            assert turn(lib, rotary(), **{name: bad}) == status
        for name in ("q", "k", "dq_out", "dk_out", "dq", "dk"):
            assert turn_back(lib, w, **{name: bad}) == status
    assert turn_back(lib, rotary(), dqw=A) == INVALID                # no such weight
    assert turn_back(lib, rotary(q_weight=A), dkw=A) == INVALID
    assert turn_back(lib, w, dqw=A + 2) == MISALIGNED and turn_back(lib, w, dkw=A + 8) == MISALIGNED
    need = lib.mra_rotary_backward_workspace_bytes(ctypes.byref(w))
    assert need > 0 and lib.mra_rotary_backward_workspace_bytes(ctypes.byref(rotary())) == 0
    assert turn_back(lib, w, dqw=A, size=need - 1) == WORKSPACE
    assert turn_back(lib, w, dqw=A, ws=None) == INVALID and turn_back(lib, w, dqw=A, ws=A + 4) == MISALIGNED


def test_rotary_empty(lib):
    none = tensor(None)
    for p in (rotary(B=0), rotary(n=0), rotary(H=0, H_kv=0)):
        assert turn(lib, p, q=none, k=none, q_out=none, k_out=none) == OK
        assert turn_back(lib, p, q=none, dq_out=none, dk_out=none, dq=none, dk=none, ws=None) == OK


BAD_CACHE = [
    (dict(pages=-1), INVALID), (dict(H_kv=-1), INVALID), (dict(B=-1), INVALID), (dict(max_pages=-1), INVALID),
    (dict(d=0), INVALID), (dict(page_size=0), INVALID), (dict(page_size=-32), INVALID), (dict(d=96), UNSUPPORTED),
    (dict(page_size=16), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=2048), UNSUPPORTED),
    (dict(H_kv=(1 << 16) + 1), UNSUPPORTED), (dict(max_pages=(1 << 21) + 1), UNSUPPORTED),
    (dict(B=1 << 22, H_kv=8), UNSUPPORTED), (dict(data=None), INVALID), (dict(table=None), INVALID),
    (dict(data=A + 8), MISALIGNED),
]


@pytest.mark.parametrize("bad,status", BAD_CACHE)
def test_caches_refused(lib, bad, status):
    c = cache(**bad)
    h = 8 if bad.get("H_kv", 2) < 2 else 4 * min(bad.get("H_kv", 2), 1 << 14)
    assert rows(lib, c) == status and rows(lib, c, read=True) == status
    assert attend(lib, c, attention(H=h, n_q=1 << 10 if "B" in bad else 5)) == status
    if status == UNSUPPORTED or status == INVALID and not {"data", "table"} & set(bad):
        assert lib.mra_fp4_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(attention(H=h, n_q=1 << 10))) == 0


def test_cache_calls_refused(lib):
    for read in (False, True):
        assert rows(lib, None, read=read) == INVALID
        assert rows(lib, cache(), n=-1, read=read) == INVALID and rows(lib, cache(), dtype=3, read=read) == UNSUPPORTED
        assert rows(lib, cache(), n=(1 << 26) + 1, read=read) == UNSUPPORTED
        assert rows(lib, cache(B=1 << 12, H_kv=1 << 10), n=1 << 10, read=read) == UNSUPPORTED
        for bad, status in BAD_TENSORS:
            assert rows(lib, cache(), k=bad, read=read) == status and rows(lib, cache(), v=bad, read=read) == status
        for c, n in ((cache(B=0), 7), (cache(H_kv=0), 7), (cache(), 0)):
            assert rows(lib, c, n=n, read=read, k=tensor(None), v=tensor(None)) == OK
    # nothing can be written to a cache without pages
    assert rows(lib, cache(pages=0, data=None), k=tensor(None)) == OK
    assert lib.mra_fp4_page_bytes(32, 64) == 32 * 68 and lib.mra_fp4_page_bytes(1024, 128) == 1024 * 136
    assert lib.mra_fp4_page_bytes(16, 64) == lib.mra_fp4_page_bytes(32, 48) == lib.mra_fp4_page_bytes(0, 0) == 0


BAD_ATTENTION = [
    (dict(H=-1), INVALID), (dict(n_q=-1), INVALID), (dict(H=7), INVALID), (dict(H=0), INVALID), (dict(scale=0.0), INVALID),
    (dict(scale=2.0 ** -65), INVALID), (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID),
    (dict(causal=2), INVALID), (dict(dtype=2), UNSUPPORTED), (dict(n_q=(1 << 26) + 1), UNSUPPORTED),
    (dict(H=(1 << 16) + 2), UNSUPPORTED), (dict(H=1 << 12, n_q=(1 << 18) // 3 + 1), UNSUPPORTED), (dict(lengths=None), INVALID),
]


@pytest.mark.parametrize("bad,status", BAD_ATTENTION)
def test_attention_refused(lib, bad, status):
    assert attend(lib, cache(), attention(**bad)) == status
    if "lengths" not in bad:
        assert lib.mra_fp4_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(attention(**bad))) == 0


def test_attention_tensors_refused(lib):
    assert attend(lib, None, attention()) == INVALID and attend(lib, cache(), None) == INVALID
    for bad, status in BAD_TENSORS:
        assert attend(lib, cache(), attention(), q=bad) == status
        assert attend(lib, cache(), attention(), out=bad) == status
    assert attend(lib, cache(), attention(), lse=A + 4) == MISALIGNED
    assert attend(lib, cache(), attention(n_q=0), q=tensor(None), out=tensor(None)) == OK
    assert attend(lib, cache(B=0), attention(), q=tensor(None), out=tensor(None)) == OK
    long = cache(max_pages=1 << 12)
    need = lib.mra_fp4_attention_workspace_bytes(ctypes.byref(long), ctypes.byref(attention(n_q=1)))
    if need:
        assert attend(lib, long, attention(n_q=1), size=need - 1) == WORKSPACE
        assert attend(lib, long, attention(n_q=1), ws=None) == INVALID
        assert attend(lib, long, attention(n_q=1), ws=A + 8) == MISALIGNED
    assert lib.mra_layer_last_hip_error() == 0


# below 2^32 threads of a launch dimension: 2^23 - 1 workgroups of 512, 2^24 - 1 of 256. What is not
# refused for its size is for a missing tensor, before anything is enqueued.
@pytest.mark.parametrize("sizes,n_q,status", [
    (dict(B=1 << 20, H_kv=8), 1, UNSUPPORTED), (dict(B=(1 << 20) - 1, H_kv=8), 1, INVALID),
    (dict(B=1 << 19, H_kv=8), 17, UNSUPPORTED), (dict(B=1 << 19, H_kv=8), 16, INVALID),
    (dict(B=1 << 16, H_kv=64), 65, INVALID), (dict(B=1 << 17, H_kv=64), 65, UNSUPPORTED),
])
def test_attention_launches_that_do_not_fit(lib, sizes, n_q, status):
    c = cache(**sizes)
    p = attention(H=c.H_kv, n_q=n_q, lengths=None)
    assert attend(lib, c, p) == status
    if status == UNSUPPORTED:
        assert lib.mra_fp4_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(p)) == 0


@pytest.mark.parametrize("B,n,status", [((1 << 21) - 1, 33, INVALID), (1 << 22, 33, UNSUPPORTED)])
def test_cache_launches_that_do_not_fit(lib, B, n, status):
    for read in (False, True):
        assert rows(lib, cache(B=B, H_kv=2), n=n, read=read, k=tensor(None)) == status


@pytest.mark.parametrize("B,n,status", [((1 << 24) - 1, 8, INVALID), (1 << 24, 8, UNSUPPORTED)])
def test_rotary_launches_that_do_not_fit(lib, B, n, status):
    assert turn(lib, rotary(B=B, n=n), q=tensor(None)) == status


def test_tensors_on_the_host_are_refused():
    q = torch.zeros(1, 2, 4, 32)
    f = ops.rotary_frequencies(32, device="cpu")
    for call in (ops.rotary, ops.rotary_forward):
        with pytest.raises(ValueError, match="ROCm device"):
            call(q, q, f)
    with pytest.raises(ValueError, match="ROCm device"):
        ops.rotary_backward(q, q, freqs=f)
    with pytest.raises(ValueError, match="either result"):
        ops.rotary_backward(None, None, freqs=f)
    c = ops.fp4_cache(2, 2, 32, 32, device="cpu")
    table = torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError, match="ROCm device"):
        ops.fp4_cache_write(c, q, q, table)
    with pytest.raises(ValueError, match="ROCm device"):
        ops.fp4_cache_read(c, table, 4)
    with pytest.raises(ValueError, match="ROCm device"):
        ops.fp4_cache_attention(q, c, table, torch.ones(1, dtype=torch.int32))
    for size, d in ((16, 64), (33, 64), (2048, 64), (32, 16), (-32, 64), (1 << 31, 64), (32, 1 << 40)):
        with pytest.raises(ValueError, match="page_size"):
            ops.fp4_cache(2, 2, size, d, device="cpu")
    for data in (torch.zeros(2, 2, 32 * 34, dtype=torch.int8), torch.zeros(2, 2, 32 * 34 + 1, dtype=torch.uint8),
                 torch.zeros(2, 32 * 34, dtype=torch.uint8), torch.zeros(2, 2, 64 * 34, dtype=torch.uint8)[..., ::2]):
        with pytest.raises(ValueError, match="contiguous uint8"):
            ops.Fp4Cache(data, 32, 32)


def test_frequencies():
    f = ops.rotary_frequencies(64, device="cpu")
    assert f.dtype == torch.float64 and f.shape == (32,) and f[0] == 1 and math.isclose(f[16], 0.01, rel_tol=1e-14)
    assert torch.equal(ops.rotary_frequencies(64, scaling="linear", factor=4.0, device="cpu"), f / 4)
    n = ops.rotary_frequencies(64, scaling="ntk", factor=8.0, device="cpu")
    assert n[0] == 1 and math.isclose(n[-1], f[-1] / 8, rel_tol=1e-12)
    b = ops.rotary_frequencies(64, scaling="by_parts", factor=8.0, original=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(b[turns >= 32], f[turns >= 32]) and torch.allclose(b[turns <= 1], f[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and bool(((b < f) & (b > f / 8))[mid].all()) and bool((b[1:] <= b[:-1]).all())
    assert len(ops.rotary_frequencies(0, device="cpu")) == 0
    assert ops.rotary_magnitude(1.0) == 1.0 and math.isclose(ops.rotary_magnitude(math.e), 1.1)
    for bad in (dict(rotary_dim=20), dict(rotary_dim=-16), dict(rotary_dim=32, base=1.0), dict(rotary_dim=32, factor=0.0),
                dict(rotary_dim=32, scaling="other"), dict(rotary_dim=32, scaling="by_parts")):
        with pytest.raises(ValueError):
            ops.rotary_frequencies(**bad, device="cpu")


def test_oracle_turns_by_hand():
    x = torch.tensor([1.0, 2.0, 3.0, 4.0] + [0.0] * 28).view(1, 1, 1, 32)
    f = torch.tensor([math.pi / 2, math.pi], dtype=torch.float64)      # quarter and half turns at position 1
    p = torch.tensor([1])
    half = L.turn(x, f, p)[0, 0, 0, :4]
    assert torch.allclose(half, torch.tensor([-3.0, -2.0, 1.0, -4.0], dtype=torch.float64))
    inter = L.turn(x, f, p, interleaved=True)[0, 0, 0, :4]
    assert torch.allclose(inter, torch.tensor([-2.0, 1.0, -3.0, -4.0], dtype=torch.float64))
    assert torch.allclose(L.turn(L.turn(x, f, p), f, p, back=True), x.double())


def test_oracle_gradients_are_autograds():
    gen = torch.Generator().manual_seed(1)
    x, g = (torch.randn(2, 3, 5, 32, generator=gen, dtype=torch.float64) for _ in range(2))
    w = torch.randn(32, generator=gen, dtype=torch.float64)
    f = ops.rotary_frequencies(16, device="cpu")
    for inter in (False, True):
        a, b = x.clone().requires_grad_(True), w.clone().requires_grad_(True)
        want = torch.autograd.grad(L.rotary(a, f, b, 1e-6, interleaved=inter, magnitude=1.3), (a, b), g)
        got = L.rotary_grads(g, x, f, w, 1e-6, interleaved=inter, magnitude=1.3)
        assert all(torch.allclose(s, t, rtol=1e-12, atol=1e-12) for s, t in zip(got, want))


def test_oracle_holds_by_hand():
    x = torch.zeros(32, dtype=torch.float64)
    x[:14] = torch.tensor([7.0, 0.24, 0.25, 0.26, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.1, -5.0, -0.3, 6.9])
    h, e = L.held(x)
    assert e.tolist() == [0]
    assert h[:14].tolist() == [6, 0, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -4, -0.5, 6]
    x[0] = 7.01                                          # above 7 steps of 1: the step is 2
    h, e = L.held(x)
    assert e.tolist() == [1] and h[:4].tolist() == [8, 0, 0, 0] and h[4] == 1.0
    for top in (2.0 ** -140, 0.0):
        assert L.held(torch.full((32,), top, dtype=torch.float64))[1].tolist() == [-125]
    h, e = L.held(torch.full((32,), 3e38, dtype=torch.float64))
    assert e.tolist() == [125] and h[0] == 6 * 2.0 ** 125
    # no value is off by more than half the distance of its neighbours
    v = torch.randn(4000, 32, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    h, e = L.held(v)
    y = v / torch.exp2(e.double())
    dist = torch.where(y.abs() < 2, 0.25, torch.where(y.abs() < 4, 0.5, 1.0))
    assert bool(((v - h).abs() <= dist * torch.exp2(e.double())).all())


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("size", [32, 64, 1024])
def test_what_a_tile_addresses_lies_in_its_page(d, size):
    """The byte ranges of the kernels' loads and stores of a tile of 32 tokens at the last place of a page."""
    nb = d // 32
    total = size * (d + d // 16)
    assert total == ops.fp4_page_bytes(size, d) and total % 16 == 0
    slot = size - 32
    codes, steps = (0, size * (d // 2)), (size * d, size * (d + nb))
    ends = (codes[1], steps[0], steps[1], total)
    for x in (0, 1):
        assert codes[x] + (slot + 31) * (d // 2) + (d // 8 - 1) * 4 + 4 <= ends[x]          # write, read: a dword
        assert codes[x] + (slot + 31) * (d // 2) + (nb - 1) * 16 + 16 <= ends[x]            # many rows: 16 bytes
        assert codes[x] + (slot + 31) * (d // 2) + 3 * (d // 8) + d // 8 <= ends[x]         # few rows: d / 8 bytes
        assert steps[x] + (slot + 31) * nb + nb - 1 < ends[2 + x]
        assert codes[x] % 16 == 0 and steps[x] % 16 == 0


def value_place(d, r, c):
    """ValueTile::place of fp4_attention.hip."""
    f = (r & 3) | (r >> 3 & 1) << 2 if d == 128 else (r >> 1 & 1) | (r >> 3 & 1) << 1 if d == 64 else r >> 3 & 1
    return r * 2 * d + (((c >> 4) ^ f) << 5) + (((c >> 3 & 1) ^ (r >> 2 & 1)) << 4) + (c & 4) * 2


@pytest.mark.parametrize("d", [32, 64, 128])
def test_values_come_back_transposed(d):
    """What lanes put and get in a wave's value tile: every place once, lane (g, i) of get(t) has channel
    16 t + i of rows 8 g .. 8 g + 7, whose weights the first product left in the same lane group."""
    places = [value_place(d, r, c) for r in range(32) for c in range(0, d, 4)]
    assert sorted(places) == list(range(0, 64 * d, 8))
    lds = {}
    for lane in range(64):                          # put: row 16 x + i, chunk n of eight channels
        g, i = lane >> 4, lane & 15
        for x in range(2):
            for n in range(d // 32):
                at = (value_place(d, i, g * (d // 4)) ^ 16 * n) + x * 16 * 2 * d
                for e in range(8):
                    lds[at + 2 * e] = (16 * x + i, g * (d // 4) + 8 * n + e)
    assert len(lds) == 32 * d
    for t in range(d // 16):                        # get: lane i of 16 receives element i % 4 of the 8 bytes of lane 4 k + i / 4
        for lane in range(64):
            g, i = lane >> 4, lane & 15
            for e in range(2):
                for k in range(4):
                    j = 4 * k + i // 4
                    at = value_place(d, 8 * g + 4 * e + (j >> 2), 4 * (j & 3)) ^ 32 * t
                    assert lds[at + 2 * (i % 4)] == (8 * g + 4 * e + k, 16 * t + i)
    # scores: the product's row 4 g + r of part x is the key that lane i = 4 g + r loaded
    for g in range(4):
        for x in range(2):
            for r in range(4):
                i = 4 * g + r
                assert 8 * (i >> 2) + 4 * x + (i & 3) == 8 * g + 4 * x + r


@pytest.mark.parametrize("d,threads", [(32, 256), (64, 256), (128, 256), (128, 512)])
def test_a_stage_converts_every_block_once(d, threads):
    """CacheStage::unit: each token's blocks of keys and values belong to one lane each."""
    nb, u = d // 32, 2 * d
    per = 2 if 2 * u > threads else 1
    seen = []
    for tid in range(threads):
        for n in range(per):
            t = tid % u // nb
            x = n if per == 2 else tid // u
            if x < 2:
                seen.append((x, (t & 48) | (t & 3) << 2 | (t >> 2 & 3), tid % u % nb))
    assert sorted(seen) == [(x, r, b) for x in range(2) for r in range(64) for b in range(nb)]
