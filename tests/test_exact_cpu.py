"""Exact attention without a GPU: the ABI's exports and refusals, the bucket map,
the oracle's pins, and the bounds of what the kernels address in LDS."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

from oracle import exact_oracle as E
from paper_2207_10284_amd import ops

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "mra_exact.h")
OK, INVALID, UNSUPPORTED, MISALIGNED, WORKSPACE = range(5)
A = 1 << 20            # a fake, 16-byte aligned address: never dereferenced


@pytest.fixture(scope="module")
def lib():
    return ops.load_exact()


def test_exports_are_the_header(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(mra_exact_[a-z_]+)\s*\(", text))
    assert names == set(ops.EXACT_SIGNATURES)
    if shutil.which("nm"):
        out = subprocess.run(["nm", "-D", "--defined-only", ops.EXACT_LIB_PATH], capture_output=True, text=True,
                             check=True).stdout
        funcs = {line.split()[-1] for line in out.splitlines() if len(line.split()) == 3 and line.split()[1] == "T"}
        assert {f for f in funcs if not f.startswith("_Z")} == names


def problem(**kw):
    p = ops._Problem(1, 2, 1, 40, 70, 64, 1, 0.125, 0, None, None, None, 0, None, 0, 0, None, 0)
    for n, x in kw.items():
        setattr(p, n, x)
    return p


def tensor(data=A, b=0, h=0, n=64):
    return ctypes.byref(ops._Strided(data, b, h, n))


def forward(lib, p, q=None, k=None, v=None, out=None, lse=None, ws=A, size=1 << 40):
    t = [tensor() if x is None else x for x in (q, k, v, out)]
    return lib.mra_exact_forward(ctypes.byref(p) if p else None, *t, lse, ws, size, None)


def backward(lib, p, ws=A, size=1 << 40, lse=A, dbias=None, **kw):
    names = ("q", "k", "v", "out", "dout", "dq", "dk", "dv")
    t = [kw.get(n) or tensor() for n in names]
    return lib.mra_exact_backward(ctypes.byref(p) if p else None, *t[:5], lse, *t[5:], dbias, ws, size, None)


BAD = [
    (dict(B=-1), INVALID), (dict(H=-1), INVALID), (dict(H_kv=-1), INVALID), (dict(n_q=-1), INVALID),
    (dict(n_k=-2), INVALID), (dict(d=0), INVALID), (dict(H=3, H_kv=2), INVALID), (dict(H_kv=0), INVALID),
    (dict(H=0, H_kv=1), INVALID), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID),
    (dict(scale=2.0 ** -65), INVALID), (dict(scale=2.0 ** 65), INVALID),
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(causal=2), INVALID),
    (dict(d=48), UNSUPPORTED), (dict(d=256), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED),
    (dict(n_q=(1 << 26) + 1), UNSUPPORTED), (dict(n_k=(1 << 26) + 1), UNSUPPORTED),
    (dict(B=1 << 20, H=1 << 20, H_kv=1), UNSUPPORTED), (dict(B=1 << 14, H=1 << 14, H_kv=1), UNSUPPORTED),
    (dict(key_mask=A, key_mask_stride=-1), INVALID),
    (dict(bias=A, buckets=0, bucket_map=A), INVALID), (dict(bias=A, buckets=8), INVALID),
    (dict(bias=A, buckets=8, bucket_map=A, far=-1), INVALID), (dict(bias=A, buckets=8, bucket_map=A, far=513), UNSUPPORTED),
    (dict(bias=A, buckets=1025, bucket_map=A), UNSUPPORTED), (dict(bias=A, buckets=8, bucket_map=A, bias_dtype=5), UNSUPPORTED),
]


@pytest.mark.parametrize("change,status", BAD)
def test_problems_refused(lib, change, status):
    p = problem(**change)
    assert forward(lib, p) == status and backward(lib, p) == status
    assert lib.mra_exact_forward_workspace_bytes(ctypes.byref(p)) == 0
    assert lib.mra_exact_backward_workspace_bytes(ctypes.byref(p)) == 0


def test_tensors_refused(lib):
    p = problem()
    assert forward(lib, None) == INVALID and backward(lib, None) == INVALID
    for bad, status in ((tensor(None), INVALID), (tensor(A + 8), MISALIGNED), (tensor(n=-64), INVALID),
                        (tensor(n=68), MISALIGNED), (tensor(n=1 << 24), UNSUPPORTED), (tensor(h=4), MISALIGNED), (tensor(b=12), MISALIGNED)):
        for name in ("q", "k", "v", "out"):
            assert forward(lib, p, **{name: bad}) == status, (name, status)
        for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
            assert backward(lib, p, **{name: bad}) == status, (name, status)
    assert forward(lib, p, lse=A + 4) == MISALIGNED
    assert backward(lib, p, lse=None) == INVALID and backward(lib, p, lse=A + 4) == MISALIGNED
    assert backward(lib, p, dbias=A) == INVALID                     # no bias
    b = problem(bias=A, buckets=8, bucket_map=A, far=3)
    assert backward(lib, b, dbias=A + 2) == MISALIGNED


def test_workspaces_refused(lib):
    p = problem(n_k=4096)                                           # few rows: workgroups share the keys
    need = lib.mra_exact_forward_workspace_bytes(ctypes.byref(p))
    assert need > 0
    assert forward(lib, p, size=need - 1) == WORKSPACE
    assert forward(lib, p, ws=None) == INVALID and forward(lib, p, ws=A + 1) == MISALIGNED
    need = lib.mra_exact_backward_workspace_bytes(ctypes.byref(p))
    assert need >= 2 * 40 * 4
    assert backward(lib, p, size=need - 1) == WORKSPACE
    assert backward(lib, p, ws=None) == INVALID and backward(lib, p, ws=A + 4) == MISALIGNED
    wide = problem(n_k=4096, bias=A, buckets=8, bucket_map=A, far=20)
    assert lib.mra_exact_backward_workspace_bytes(ctypes.byref(wide)) > need


def test_empty_problems(lib):
    none = tensor(None)
    for change in (dict(B=0), dict(H=0, H_kv=0), dict(n_q=0)):
        p = problem(**change)
        assert forward(lib, p, q=none, k=none, v=none, out=none, ws=None) == OK
        assert lib.mra_exact_forward_workspace_bytes(ctypes.byref(p)) == 0
    p = problem(B=0)
    assert backward(lib, p, ws=None, lse=None, q=none, k=none, v=none, out=none, dout=none, dq=none, dk=none,
                    dv=none) == OK
    assert lib.mra_exact_last_hip_error() == 0


def test_tensors_on_the_host_are_refused():
    q = torch.zeros(1, 1, 4, 32)
    for call in (ops.exact_attention, ops.exact_attention_forward):
        with pytest.raises(ValueError, match="ROCm device"):
            call(q, q, q)
    with pytest.raises(ValueError, match="ROCm device"):
        ops.exact_attention_backward(q, q, q, q, q, torch.zeros(1, 1, 4))


def test_bucket_map_by_hand():
    """Eight buckets, both directions, distance 16: 0 1, then from 2 on
    2 + floor(2 log(r / 2) / log 8): 2 for r < 2 sqrt(8), so 3 from 6 on."""
    m = ops.distance_buckets(8, 16, True, device="cpu").tolist()
    far = len(m) // 2
    assert far == 6 and m[far] == 0
    assert [m[far - r] for r in range(1, 7)] == [1, 2, 2, 2, 2, 3]
    assert [m[far + r] for r in range(1, 7)] == [5, 6, 6, 6, 6, 7]
    one = ops.distance_buckets(4, 8, False, device="cpu").tolist()   # 0 1 2 2 3: 2 sqrt(4) = 4
    assert one == [3, 2, 2, 1, 0, 0, 0, 0, 0]


@pytest.mark.parametrize("num,dist,both", [(32, 128, True), (32, 128, False), (64, 256, True), (16, 50, False), (40, 300, True)])
def test_bucket_map_formula(num, dist, both):
    """The formula in high precision away from its borders, and its monotony."""
    m = ops.distance_buckets(num, dist, both, device="cpu").tolist()
    far, n = len(m) // 2, num // 2 if both else num
    e = n // 2
    back = [m[far - r] for r in range(far + 1)]
    assert back == sorted(back) and back[-1] == n - 1 and back[-2] == n - 2
    assert [m[far + r] for r in range(1, far + 1)] == ([n + x for x in back[1:]] if both else [0] * far)
    for r in range(far + 1):
        x = r if r < e else e + (n - e) * math.log(r / e) / math.log(dist / e)
        if r < e or abs(x - round(x)) > 1e-9:
            assert back[r] == min(int(x), n - 1)


@pytest.mark.parametrize("args", [(1, 8, False), (2, 8, True), (7, 20, True), (2048, 5000, True), (8, 2, True), (4, 2, False),
                                  (32, 100000, True)])
def test_bucket_map_refused(args):
    with pytest.raises(ValueError):
        ops.distance_buckets(*args, device="cpu")


# ---------------------------------------------------------------- the oracle's pins
def _small(seed=5, B=2, H=4, Hkv=2, nq=7, nk=11, d=8):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    buckets = ops.distance_buckets(8, 16, True, device="cpu")
    return (r(B, H, nq, d), r(B, Hkv, nk, d), r(B, Hkv, nk, d), r(B, H, nq, d),
            dict(causal=True, lengths=torch.tensor([11, 6], dtype=torch.int32), key_mask=torch.rand(B, nk, generator=gen) < 0.8,
                 q_start=torch.tensor([-2, 4], dtype=torch.int32), bias=r(8, H), buckets=buckets, scale=0.4))


def test_oracle_is_the_definition():
    """Entry by entry in Python."""
    q, k, v, _, o = _small()
    Z, L, _ = E.attention(q, k, v, **o)
    far = len(o["buckets"]) // 2
    for b in range(2):
        for h in range(4):
            for i in range(7):
                p = int(o["q_start"][b]) + i
                w = {}
                for j in range(11):
                    if j < o["lengths"][b] and o["key_mask"][b, j] and j <= p:
                        s = 0.4 * float(q[b, h, i] @ k[b, h // 2, j])
                        s += float(o["bias"][o["buckets"][max(-far, min(far, j - p)) + far], h])
                        w[j] = math.exp(s)
                t = sum(w.values())
                if not w:
                    assert L[b, h, i] == -math.inf and not Z[b, h, i].any()
                    continue
                assert abs(float(L[b, h, i]) - math.log(t)) < 1e-12
                z = sum(x / t * v[b, h // 2, j] for j, x in w.items())
                assert (Z[b, h, i] - z).abs().max() < 1e-12


def test_oracle_gradients():
    """The chain rule against autograd and against differences."""
    q, k, v, g, o = _small()
    got = E.gradients(q, k, v, g, **o)
    leaves = [t.clone().requires_grad_(True) for t in (q, k, v, o["bias"])]
    z = E.attention(*leaves[:3], **{**o, "bias": leaves[3]})[0]
    for x, r in zip(got, torch.autograd.grad(z, leaves, g)):
        assert (x - r).abs().max() < 1e-12
    mag = E.gradients(q, k, v, g, absolute=True, **o)
    base = [q, k, v, o["bias"]]
    for n, (x, m) in enumerate(zip(got, mag)):
        assert (m >= x.abs() - 1e-12).all()
        step = torch.randn(base[n].shape, generator=torch.Generator().manual_seed(n), dtype=torch.float64)
        at = []
        for f in (1e-5, -1e-5):
            t = list(base)
            t[n] = t[n] + f * step
            at.append(float((E.attention(*t[:3], **{**o, "bias": t[3]})[0] * g).sum()))
        assert abs((at[0] - at[1]) / 2e-5 - float((x * step).sum())) < 1e-7


# ---------------------------------------------------------------- what the kernels address
PAD = 64


@pytest.mark.parametrize("far", [0, 1, 2, 31, 91, 512])
def test_bias_window_covers_every_near_tile(far):
    """A tile that is not on one side of +-far reads and adds to the window's
    2 far + 128 entries at far + 64 + distance, for each of its 63 distances."""
    entries = 2 * far + 2 * PAD
    for d0 in range(-far - 40, far + 41):                           # key 0 - query 0
        low, high = d0 + 31 <= -far, d0 - 31 >= far
        rels = [d0 + kk - qq for kk in (0, 31) for qq in (0, 31)]
        if low:
            assert max(rels) <= -far
        elif high:
            assert min(rels) >= far
        else:
            at = [r + far + PAD for r in rels]
            assert 0 <= min(at) and max(at) < entries
            for x in range(min(at), max(at) + 1):                   # and the window holds that distance's entry
                assert min(max(x - PAD, 0), 2 * far) == min(max(x - far - PAD, -far), far) + far


def test_skewed_tile():
    """Query q's key k goes to row q, column k - q + 31 of 32 x 64 floats; the
    addresses of a near tile's 64 columns in the window stay inside it."""
    seen = {63 * q + 31 + k: (q, k) for q in range(32) for k in range(32)}
    assert len(seen) == 1024 and all(divmod(x, 64) == (q, k - q + 31) for x, (q, k) in seen.items())
    for far in (0, 1, 91, 512):
        for d0 in range(-far - 30, far + 31):
            assert 0 <= d0 + far + PAD - 31 and d0 + far + PAD - 31 + 63 < 2 * far + 2 * PAD


@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("rows,threads", [(64, 256), (32, 256), (32, 64)])
def test_stage_writes_each_chunk_once(d, rows, threads):
    """The units of Stage cover the rows' eight-element chunks once, each inside
    its tile, and a lane's operand reads find them there."""
    if rows * (d // 8) % threads or rows * (d // 8) < threads:
        pytest.skip("not a stage of this width")
    swz = {128: lambda r: 4 * (r & 3) + ((r >> 2) & 3), 64: lambda r: 4 * ((r >> 1) & 1) + ((r >> 2) & 3),
           32: lambda r: (r >> 2) & 3}[d]
    off = lambda r, c: r * 2 * d + (((2 * c >> 4) ^ swz(r)) << 4) + (2 * c & 15)
    at = {}
    cpr = d // 8
    for i in range(rows * cpr // threads):
        for tid in range(threads):
            u = i * threads + tid
            r, c = u // cpr, 8 * (u % cpr)
            x = (r >> 5) * 64 * d + off(r & 31, c)
            assert x not in at and 0 <= x <= rows * 2 * d - 16
            at[x] = (r, c)
    assert len(at) == rows * cpr
    for lane in range(64):
        h, j = lane >> 5, lane & 31
        for c in range(d // 16):
            assert at[off(j, d // 2 * h + 8 * c)] == (j, d // 2 * h + 8 * c)


def swz(d, r):
    return 4 * (r & 3) + ((r >> 2) & 3) if d == 128 else (4 * ((r >> 1) & 1) + ((r >> 2) & 3) if d == 64 else (r >> 2) & 3)


def test_few_addresses():
    """d = 128: a lane's row chunk c and its transposed column tile t sit at the
    first's address exclusive-or 16 c and 64 t."""
    off = lambda r, c: r * 256 + (((2 * c >> 4) ^ swz(128, r)) << 4) + (2 * c & 15)
    for lane in range(64):
        h, j, i16 = lane >> 5, lane & 31, lane & 15
        for c in range(8):
            assert off(j, 64 * h + 8 * c) == off(j, 64 * h) ^ 16 * c
        for e in range(2):
            r, c0 = 4 * h + i16 // 4 + 8 * e, 16 * ((lane >> 4) & 1) + 4 * (i16 & 3)
            for t in range(4):
                assert off(r, 32 * t + c0) == off(r, c0) ^ 64 * t


@pytest.mark.parametrize("elem,d,rows,threads", [(2, 32, 64, 256), (2, 64, 64, 256), (2, 128, 64, 256), (4, 32, 64, 256),
                                                 (4, 64, 32, 256), (4, 128, 32, 256), (2, 128, 32, 64), (4, 32, 32, 64)])
def test_stage_buffers_end_with_the_last_row(elem, d, rows, threads):
    """The loads of a unit's buffer are in its range exactly for the rows that
    count (range: the last such row's end), for rows side by side and apart."""
    cpr, loads = d // 8, elem // 2
    per = threads // cpr
    for stride in (d * elem, 3 * d * elem, (1 << 25) - 16):
        for left in (1, 2, 31, 32, 33, 63, 64, 100):
            for i in range(rows * cpr // threads):
                n = min(left - i * per, per)
                size = (n - 1) * stride + cpr * loads * 16 if n > 0 else 0
                assert size < 1 << 32
                for tid in {0, 1, cpr - 1, cpr, threads // 2, threads - 1} | {max(0, min(n, per - 1)) * cpr}:
                    for e in range(loads):
                        at = tid // cpr * stride + tid % cpr * loads * 16 + 16 * e
                        assert at + 16 < 1 << 32
                        assert (at + 16 <= size) == (i * per + tid // cpr < left)


def head_block(p, heads, blocks, causal):
    rest = heads % 8
    whole = (heads - rest) * blocks
    if p < whole:
        q, r = divmod(p, 8 * blocks)
        return 8 * q + r % 8, r // 8
    r = p - whole
    if causal:
        return heads - rest + r % rest, r // rest
    total = rest * blocks
    x, slot, q, m = r % 8, r // 8, total // 8, total % 8
    x = x * (q + 1) + slot if x < m else m * (q + 1) + (x - m) * q + slot
    return heads - rest + x // blocks, x % blocks


@pytest.mark.parametrize("causal", [False, True])
def test_head_blocks_are_each_taken_once(causal):
    for heads in (1, 3, 7, 8, 9, 12, 96):
        for blocks in (1, 2, 5, 13, 64):
            got = {head_block(p, heads, blocks, causal) for p in range(heads * blocks)}
            assert got == {(h, b) for h in range(heads) for b in range(blocks)}


def test_parts_cover_every_stage_once():
    """Ranges of the stages of all heads, head after head (dK, dV)."""
    for group in (1, 3, 8):
        for stages in (0, 1, 2, 7, 40):
            for parts in (1, 2, 6, 8):
                seen = []
                for part in range(parts):
                    t0, t1 = group * stages * part // parts, group * stages * (part + 1) // parts
                    hg = t0 // stages if stages else group
                    while hg < group and hg * stages < t1:
                        seen += [(hg, st) for st in range(max(t0 - hg * stages, 0), min(t1 - hg * stages, stages))]
                        hg += 1
                assert seen == [(h, st) for h in range(group) for st in range(stages)]


def test_number_chunk():
    """hi + mid + lo, each the rest rounded to bfloat16, are the number to 2^-24."""
    x = torch.cat([torch.randn(1000, generator=torch.Generator().manual_seed(1)) * 10.0 ** e for e in range(-3, 6)])
    x = torch.cat([x, torch.tensor([0.0, -3e38, 1e-20])])
    hi = x.bfloat16().float()
    mid = (x - hi).bfloat16().float()
    lo = (x - hi - mid).bfloat16().float()
    assert ((hi.double() + mid + lo - x).abs() <= 2.0 ** -24 * x.abs()).all()


def test_lds_fits():
    """Dynamic LDS of every launch, at the widest window, within 160 KB."""
    for planes, d in ((p, d) for p in (1, 3) for d in (32, 64, 128)):
        rows = 64 if planes == 1 or d == 32 else 32
        stage = 4 * planes * rows * d * 2
        win = (2 * 512 + 2 * PAD) * 4
        assert stage + 5 * win + 4 * 32 * 64 * 4 <= 160 * 1024      # dQ: the bias, four windows of sums and skewed tiles
        assert stage + 64 * rows + win <= 160 * 1024                # dK, dV
        assert max(4 * planes * 32 * d * 2, 3 * 32 * d * 4) + 2048 <= 160 * 1024


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("causal", [False, True])
def test_walk_of_dk_dv(bias, causal):
    """The walk of dK and dV from the last query down, as exact_dkv_kernel makes it: every
    stage of every head once over the parts, none before the first query that reaches a key,
    and the stages taken as plain have only queries that reach every key of the block."""
    QT, rows = 64, 128
    for group, nq, nk, start, block0, parts in ((1, 1, 1, 0, 0, 1), (3, 300, 200, -100, 128, 1), (4, 1000, 1000, 0, 384, 4),
                                                (2, 700, 1500, 800, 1408, 3), (8, 65, 500, 900, 256, 8), (2, 0, 90, 0, 0, 2),
                                                (4, 130, 130, -500, 0, 2), (1, 640, 640, 0, 512, 6)):
        first = min(max(block0 - start, 0), nq) // QT * QT if causal else 0
        stages = (nq - first + QT - 1) // QT if block0 < nk else 0
        border = min(max(block0 + rows - 1 - start - first + QT - 1, 0) // QT, stages) if causal else 0
        inner = 1 if bias else group
        turn, total, seen = inner * stages, group * stages, []
        for part in range(parts):
            t0, t1 = total * part // parts, total * (part + 1) // parts
            hg = group if stages == 0 else t0 // turn * inner
            while hg < group and hg * stages < t1:
                begin, end = max(t0 - hg * stages, 0), min(t1 - hg * stages, turn)
                plain = begin + (max(min((stages - border) * inner, end) - begin, 0) & ~1)
                q, hn = first + (stages - 1 - begin // inner) * QT, begin % inner
                for st in range(begin, end):
                    seen.append((hg + hn, q))
                    if st < plain:
                        assert not causal or start + q >= block0 + rows - 1
                    if st + 1 < end:
                        hn += 1
                        if hn == inner:
                            hn, q = 0, q - QT
                hg += inner
        want = [(h, q) for h in range(group) for q in range(first, nq, QT)] if block0 < nk else []
        assert sorted(seen) == want
