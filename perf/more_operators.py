"""Rotary positions, norms of queries and keys with the rotation in the same pass, a cache held in 4
bits (written, read back) and attention over it, as measurable cases.

``op`` "rotary": queries and keys rotated, at position p, pair (a, b) of frequency f by the angle p f:

    a' = m (a cos - b sin)      b' = m (b cos + a sin)

with, where ``norm``, x (mean x^2 + eps)^-1/2 w of each head's row in the place of x. Pairs are elements i
and i + r/2 ("half") or 2i and 2i + 1 of the first r elements of a row; the rest is not rotated.
``mode`` "train" returns the results and the gradients of queries, keys and weights.

``op`` "write": new keys and values written to a paged cache and read back; "read": read back only. A
block of 32 channels of a token shares s = 2^e, the smallest power of two (-125 <= e <= 125) with max |x| <= 7 s;
x / s is held as the nearest of +-{0, 1/2, 1, 3/2, 2, 3, 4, 6}, ties to the even one in this order.

``op`` "attend": softmax(scale q k^T) v over the values the cache holds; query i of sequence b stands at
position length_b - nq + i, keys before the length count, in causal calls up to the position. Query head h
reads key head h // (H / Hkv).
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-6


def _rotary(name, mode, dtype, B, H, Hkv, n, d, rot, pairs="half", norm=False, base=10000.0, scaling="none",
            factor=1.0, original=0, places="first", layout="bnhd"):
    c = dict(op="rotary", mode=mode, dtype=dtype, B=B, H=H, Hkv=Hkv, n=n, d=d, rot=rot, pairs=pairs, norm=norm,
             base=base, scaling=scaling, factor=factor, original=original, places=places, layout=layout)
    return dict(c, name=name) if name else c


def _cache(name, op, dtype, B, H, Hkv, nq, nk, d, page, causal=False, ragged=True, layout="bnhd"):
    """``nq``: new tokens (write), queries (attend); ``nk``: the longest sequence."""
    c = dict(op=op, dtype=dtype, B=B, H=H, Hkv=Hkv, nq=nq, nk=nk, d=d, page=page, causal=causal, ragged=ragged,
             layout=layout)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token for each of 32 served sequences, twelve heads; latency
        _rotary("rotary-token", "infer", "bf16", 32, 12, 12, 1, 64, 64, places="ragged"),
        # a RoBERTa-base-sized layer at 4096 tokens, training on views of one projection's output
        _rotary("rotary-base-4096-train", "train", "bf16", 8, 12, 12, 4096, 64, 64, layout="qkv"),
        # half of the head rotated, interleaved pairs, float32, an odd length at far positions, a raised base
        _rotary("rotary-far-2999", "infer", "f32", 4, 8, 2, 2999, 128, 64, "interleaved", scaling="ntk", factor=8.0,
                places="far", layout="bhnd"),
        # one new token for each of four long sequences, queries and keys normalised; latency
        _rotary("norm-rotary-token", "infer", "bf16", 4, 16, 4, 1, 128, 128, norm=True, scaling="by_parts", factor=8.0,
                original=4096, places="ragged"),
        # 32768 tokens, 16 heads of width 128 on four key heads, scaled from a context of 4096, training
        _rotary("norm-rotary-32768-train", "train", "bf16", 1, 16, 4, 32768, 128, 128, norm=True, scaling="by_parts",
                factor=8.0, original=4096),
        # one new token of 32 sequences into their caches of up to 4096, twelve heads; latency
        _cache("write-token", "write", "bf16", 32, 12, 12, 1, 4096, 64, 64),
        # prompts of up to 4096 tokens written at once, from views of one projection's output, and read back
        _cache("write-4096", "write", "bf16", 8, 12, 12, 4096, 4096, 64, 64, layout="qkv"),
        # four long caches read back, as for a pass that needs them whole
        _cache("read-32768", "read", "bf16", 4, 16, 4, 0, 32768, 128, 256),
        # one new token for each of 32 sequences against caches of up to 4096 keys, twelve heads
        _cache("attend-token-4096", "attend", "bf16", 32, 12, 12, 1, 4096, 64, 64, True),
        # one new token against few long caches, four query heads to a key head
        _cache("attend-token-32768", "attend", "bf16", 4, 16, 4, 1, 32768, 128, 256, True),
        # float32 queries of an odd length on an odd cache of small pages, head width 32
        _cache("attend-333-1501", "attend", "f32", 4, 8, 2, 333, 1501, 32, 32, True, layout="bhnd"),
        # the last 512 tokens of two prompts of up to 16384, processed in pieces (the largest)
        _cache("attend-512-16384", "attend", "bf16", 2, 16, 4, 512, 16384, 128, 128, True),
    ]


def _pairs(c):
    """Query-key pairs that count, ragged sequences by their mean share."""
    mean = c["nk"] * (0.75 if c["ragged"] else 1.0)
    return c["B"] * c["H"] * c["nq"] * max(mean - (c["nq"] / 2 if c["causal"] else 0), mean / 2)


def _cost(c):
    """Rough microseconds of a plain pass' bytes and products."""
    w = work(c)
    extra = 6 * c["B"] * c["H"] * c["nq"] * c["nk"] * 4 if c["op"] == "attend" else 0
    gathered = 4 * c["B"] * c["Hkv"] * c["nk"] * c["d"] * 4 if c["op"] in ("attend", "read") else 0
    return (w["bytes"] + extra + gathered) / 4e6 + w["flops"] / 1e8


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    top = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["rotary", "rotary", "rotary", "write", "read", "attend", "attend", "attend"])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        d = rng.choice([32, 64, 64, 128, 128])
        B, Hkv = _log(rng, 1, 48), rng.choice([1, 2, 3, 4, 8, 12])
        H = Hkv * rng.choice([1, 1, 2, 4, 8])
        if op == "rotary":
            n = 1 if rng.random() < 0.2 else _log(rng, 2, 32768)
            rot = rng.choice([r for r in (d, d, d // 2, d // 4) if r >= 16])
            scaling = rng.choice(["none", "none", "linear", "ntk", "by_parts"])
            c = _rotary("", rng.choice(["infer", "train"]), dtype, B, H, Hkv, n, d, rot,
                        rng.choice(["half", "half", "interleaved"]), rng.random() < 0.5,
                        rng.choice([10000.0, 10000.0, 500000.0]), scaling,
                        1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.0, 32.0]),
                        rng.choice([512, 4096]) if scaling == "by_parts" else 0,
                        rng.choice(["first", "ragged", "far"]), rng.choice(["bhnd", "bnhd", "qkv"] if H == Hkv else ["bhnd", "bnhd"]))
            elems = B * (H + 2 * Hkv) * n * d
        else:
            nk = _log(rng, 16, 32768)
            if op == "write":
                nq = rng.choice([1, 1, nk, _log(rng, 1, nk)])
            elif op == "read":
                nq = 0
            else:
                nq = min(nk, rng.choice([1, 1, 1, 2, 5, _log(rng, 8, 1024)]))
            page = rng.choice([32, 64, 64, 128, 256])
            c = _cache("", op, dtype, B, H, Hkv, nq, nk, d, page, rng.random() < 0.8, rng.random() < 0.8,
                       rng.choice(["bhnd", "bnhd"]))
            elems = B * (2 * Hkv * nk + H * nq) * d
        if _cost(c) <= top and elems <= 1 << 28:
            return c


def _dtype(c):
    return torch.bfloat16 if c["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(220710284 + seed)
    return gen


def _rows(c, gen, heads, n, spread=False):
    """[B, heads, n, d] in the case's layout; ``spread``: channels of unlike size, some of them large, as keys have."""
    B, d, dt = c["B"], c["d"], _dtype(c)
    x = torch.randn((B, n, heads, d) if c["layout"] != "bhnd" else (B, heads, n, d), generator=gen, device="cuda")
    if spread:
        size = torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda"))
        x = x * torch.where(torch.rand(d, generator=gen, device="cuda") < 0.03, 6.0 * size, size)
    x = x.to(dt)
    return x if c["layout"] == "bhnd" else x.transpose(1, 2)


def _rotary_inputs(c, seed):
    gen = _generator(seed)
    B, H, Hkv, n, d, dt = c["B"], c["H"], c["Hkv"], c["n"], c["d"], _dtype(c)
    if c["layout"] == "qkv":                    # views of one projection's output
        q, k, _ = (t.transpose(1, 2) for t in torch.randn(B, n, 3, H, d, generator=gen, device="cuda").to(dt).unbind(2))
    else:
        q, k = _rows(c, gen, H, n), _rows(c, gen, Hkv, n)
    s = dict(q=q, k=k, gq=None, gk=None, wq=None, wk=None)
    if c["mode"] == "train":
        s["gq"], s["gk"] = _rows(c, gen, H, n), _rows(c, gen, Hkv, n)
    if c["norm"]:
        s["wq"], s["wk"] = ((1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) for _ in range(2))
    first = torch.zeros(B, 1, dtype=torch.int64, device="cuda")
    if c["places"] == "ragged":                 # sequences that have come to different lengths
        first = torch.randint(0, 32768, (B, 1), generator=gen, device="cuda")
    if c["places"] == "far":                    # about a million tokens in
        first = torch.randint(900000, 1100000, (B, 1), generator=gen, device="cuda")
    s["positions"] = (first + torch.arange(n, device="cuda")).to(torch.int32)
    return s


def _frequencies(c):
    """base^(-2i/r), float64; "linear": divided by the factor; "ntk": of a base raised so that the slowest
    is divided by the factor; "by_parts": those that turn fewer than once within the original context are divided by
    it, those of more than 32 turns stay, and in between the two are mixed linearly in the turns."""
    r, base, factor = c["rot"], c["base"], c["factor"]
    if c["scaling"] == "ntk":
        base *= factor ** (r / (r - 2))
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    if c["scaling"] == "linear":
        f = f / factor
    if c["scaling"] == "by_parts":
        keep = ((c["original"] * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f / factor * (1 - keep) + f * keep
    return f


def _magnitude(c):
    return 0.1 * math.log(c["factor"]) + 1 if c["scaling"] == "by_parts" else 1.0


def _cache_inputs(c, seed):
    """Keys and values (all of the sequences' for read and attend, the new ones for write), queries, the page
    table, lengths, and for write where the new tokens begin and how many there are."""
    gen = _generator(seed)
    B, H, Hkv, nq, nk, page = (c[x] for x in ("B", "H", "Hkv", "nq", "nk", "page"))
    n = nq if c["op"] == "write" else nk
    if c["layout"] == "qkv":
        _, k, v = (t.transpose(1, 2) for t in
                   torch.randn(B, n, 3, H, c["d"], generator=gen, device="cuda").to(_dtype(c)).unbind(2))
    else:
        k, v = _rows(c, gen, Hkv, n, True), _rows(c, gen, Hkv, n)
    s = dict(k=k, v=v, q=None, starts=None, counts=None, nk=nk, n=n)
    most = -(-nk // page)
    s["pages"] = B * most + 3
    s["table"] = torch.randperm(s["pages"], generator=gen, device="cuda")[: B * most].view(B, most).to(torch.int32)
    lo = max(nk // 2, nq, 1) if c["ragged"] else nk
    s["lengths"] = torch.randint(lo, nk + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    if c["op"] == "attend":
        s["q"] = _rows(c, gen, H, nq)
    if c["op"] == "write":                      # ragged prompts, or the last tokens of ragged sequences
        if nq * 2 > nk:
            s["counts"] = s["lengths"].clamp(max=nq)
            s["starts"] = torch.zeros_like(s["lengths"])
        else:
            s["counts"] = torch.full_like(s["lengths"], nq)
            s["starts"] = s["lengths"] - nq
    return s


def prepare(case, seed):
    c = case
    if c["op"] == "rotary":
        s = _rotary_inputs(c, seed)
        s.update(op="rotary", train=c["mode"] == "train", interleaved=c["pairs"] == "interleaved", magnitude=_magnitude(c))
        if own:
            from paper_2207_10284_amd import ops
            s["freqs"] = ops.rotary_frequencies(c["rot"], c["base"], scaling=None if c["scaling"] == "none" else c["scaling"],
                                                factor=c["factor"], original=c["original"] or None, device="cuda")
        else:
            s["freqs"] = _frequencies(c).to("cuda")
        if s["train"]:
            for name in ("q", "k", "wq", "wk"):
                if s[name] is not None:
                    s[name].requires_grad_(True)
        return s
    s = _cache_inputs(c, seed)
    s.update(op=c["op"], dtype=_dtype(c), causal=c["causal"])
    if own:
        from paper_2207_10284_amd import ops
        s["cache"] = ops.fp4_cache(s["pages"], c["Hkv"], c["page"], c["d"], device="cuda")
        if c["op"] != "write":
            ops.fp4_cache_write(s["cache"], s["k"], s["v"], s["table"], counts=s["lengths"])
    else:
        s["cache"] = {}
        for name in ("k", "v"):
            shape = s["pages"], c["Hkv"], c["page"]
            s["cache"][name] = (torch.zeros(*shape, c["d"] // 2, dtype=torch.uint8, device="cuda"),
                                torch.zeros(*shape, c["d"] // 32, dtype=torch.uint8, device="cuda"))
            if c["op"] != "write":
                _store(s["cache"][name], s[name], s["table"], torch.zeros_like(s["lengths"]), s["lengths"])
    if c["op"] != "write":
        s["k"] = s["v"] = None                  # a decoder keeps the cache only
    return s


def run(state):
    s = state
    if not own:
        with torch.no_grad():
            return {"rotary": _plain_rotary, "write": _plain_write, "read": _plain_read, "attend": _plain_attend}[s["op"]](s)
    from paper_2207_10284_amd import ops
    if s["op"] == "rotary":
        args = dict(positions=s["positions"], interleaved=s["interleaved"], magnitude=s["magnitude"], q_weight=s["wq"],
                    k_weight=s["wk"], eps=EPS)
        if not s["train"]:
            return ops.rotary_forward(s["q"], s["k"], s["freqs"], **args)
        yq, yk = ops.rotary(s["q"], s["k"], s["freqs"], **args)
        leaves = [s[x] for x in ("q", "k", "wq", "wk") if s[x] is not None]
        return (yq.detach(), yk.detach(), *torch.autograd.grad((yq, yk), leaves, (s["gq"], s["gk"])))
    if s["op"] == "write":
        ops.fp4_cache_write(s["cache"], s["k"], s["v"], s["table"], starts=s["starts"], counts=s["counts"])
        return ops.fp4_cache_read(s["cache"], s["table"], s["n"], starts=s["starts"], counts=s["counts"], dtype=s["dtype"])
    if s["op"] == "read":
        return ops.fp4_cache_read(s["cache"], s["table"], s["n"], counts=s["lengths"], dtype=s["dtype"])
    return ops.fp4_cache_attention(s["q"], s["cache"], s["table"], s["lengths"], causal=s["causal"])


def _plain_rotary(s):
    r = 2 * len(s["freqs"])
    angle = s["positions"].double()[:, None, :, None] * s["freqs"]
    cos, sin = ((f(angle) * s["magnitude"]).float() for f in (torch.cos, torch.sin))

    def turn(x, sin):
        if s["interleaved"]:
            a, b = x[..., 0:r:2], x[..., 1:r:2]
            y = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = x[..., : r // 2], x[..., r // 2: r]
            y = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((y, x[..., r:]), -1)

    results, grads, wgrads = [], [], []
    for x, w, g in ((s["q"], s["wq"], s["gq"]), (s["k"], s["wk"], s["gk"])):
        f = x.float()
        if w is not None:
            inv = ((f * f).mean(-1, keepdim=True) + EPS).rsqrt()
            f = f * inv
        results.append(turn(f if w is None else f * w.float(), sin).to(x.dtype))
        if g is not None:
            back = turn(g.float(), -sin)
            if w is not None:
                wgrads.append((back * f).sum((0, 1, 2), dtype=torch.float64).to(w.dtype))
                back = back * w.float()
                back = inv * (back - f * (back * f).mean(-1, keepdim=True))
            grads.append(back.to(x.dtype))
    return (*results, *grads, *wgrads)


def _places(table, page, starts, counts, n):
    """Pages and slots [B, n] of the tokens starts + i, and which i < counts."""
    i = torch.arange(n, device=table.device)
    at = (starts.long()[:, None] + i).clamp(max=table.shape[1] * page - 1)
    return table.long().gather(1, at // page), at % page, i < counts[:, None]


def _store(held, x, table, starts, counts):
    """Codes and scales of x [B, heads, n, d] into the pages. A code is the number of borders that |x| / s
    is past (at or past, where the even neighbour is above), plus 8 for negative ones."""
    codes, scales = held
    page, (B, heads, n, d) = codes.shape[2], x.shape
    f = x.float().reshape(B, heads, n, d // 32, 32)
    top = f.abs().amax(-1, keepdim=True)
    m, e = torch.frexp(top)                     # top = m 2^e, m in [0.5, 1): 7 s = 0.875 * 2^3 s
    e = torch.where(top > 0, e - 3 + (m > 0.875).int(), -125).clamp(-125, 125)
    y = torch.ldexp(f, -e)
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for border, even_above in ((0.25, 0), (0.75, 1), (1.25, 0), (1.75, 1), (2.5, 0), (3.5, 1), (5.0, 0)):
        code += (a >= border if even_above else a > border).to(torch.uint8)
    code = code + (y < 0).to(torch.uint8) * 8
    code = code.view(B, heads, n, d)
    pages, slots, live = _places(table, page, starts, counts, n)
    b, i = live.nonzero(as_tuple=True)
    codes[pages[b, i], :, slots[b, i]] = (code[..., 0::2] | code[..., 1::2] << 4)[b, :, i]
    scales[pages[b, i], :, slots[b, i]] = (e[..., 0] + 127).to(torch.uint8)[b, :, i]


def _load(held, table, starts, counts, n):
    """The values [B, heads, n, d] that the pages hold for the tokens starts + i; 0 from counts on."""
    codes, scales = held
    pages, slots, live = _places(table, codes.shape[2], starts, counts, n)
    packed, e = codes[pages, :, slots], scales[pages, :, slots]          # [B, n, heads, d / 2], [.., d / 32]
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=codes.device)
    code = torch.stack((packed & 15, packed >> 4), -1).flatten(-2).int()
    x = grid[code & 7] * (1 - 2 * (code >> 3)).float()
    x = torch.ldexp(x.unflatten(-1, (-1, 32)), e.int()[..., None] - 127).flatten(-2)
    return torch.where(live[:, :, None, None], x, 0.0).transpose(1, 2)


def _plain_read(s):
    starts = torch.zeros_like(s["lengths"]) if s["starts"] is None else s["starts"]
    counts = s["lengths"] if s["counts"] is None else s["counts"]
    return tuple(_load(s["cache"][x], s["table"], starts, counts, s["n"]).to(s["dtype"]) for x in ("k", "v"))


def _plain_write(s):
    for x in ("k", "v"):
        _store(s["cache"][x], s[x], s["table"], s["starts"], s["counts"])
    return _plain_read(s)


def _plain_attend(s):
    q, nk, lengths = s["q"], s["nk"], s["lengths"]
    B, H, nq, d = q.shape
    zero = torch.zeros_like(lengths)
    out = torch.empty(B, H, nq, d, dtype=q.dtype, device=q.device)
    Hkv = s["cache"]["k"][0].shape[1]
    group = H // Hkv
    step = max(1, min(B, (1 << 28) // (H * nk * max(nq, d))))           # sequences at once
    key = torch.arange(nk, device=q.device)
    for b0 in range(0, B, step):
        b = slice(b0, min(B, b0 + step))
        K, V = (_load(s["cache"][x], s["table"][b], zero[b], lengths[b], nk) for x in ("k", "v"))
        Q = q[b].float().reshape(-1, Hkv, group * nq, d)                # a key head's queries, head by head
        S = (Q @ K.transpose(2, 3)).mul_(d ** -0.5).view(-1, H, nq, nk)
        keep = key < lengths[b, None, None]
        if s["causal"]:
            at = lengths[b, None].long() - nq + torch.arange(nq, device=q.device)
            keep = keep & (key <= at[:, :, None])
        S.masked_fill_(~keep[:, None], -math.inf)
        top = S.amax(-1, keepdim=True)
        P = S.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
        total = P.sum(-1, keepdim=True)
        Z = P.view(-1, Hkv, group * nq, nk) @ V
        Z = Z.view(-1, H, nq, d) / torch.where(total == 0, 1.0, total)
        out[b] = Z.to(q.dtype)
    return out


def work(case):
    c = case
    elem = 2 if c["dtype"] == "bf16" else 4
    if c["op"] == "rotary":
        values = c["B"] * (c["H"] + c["Hkv"]) * c["n"] * c["d"]
        train = c["mode"] == "train"
        # in and out; training: the results' gradients in and the inputs' out as well (without a norm
        # the gradients need no queries or keys). Three operations a rotated value, five a normalised one (ten backward)
        flops = 3 * values * c["rot"] / c["d"] * (2 if train else 1) + (5 + 10 * train) * values * c["norm"]
        return {"bytes": values * elem * (4 if train else 2), "flops": flops}
    held = c["d"] * 17 / 16                                              # bytes of a token's key and value
    share = 0.75 if c["ragged"] else 1.0
    if c["op"] == "write":
        tokens = c["B"] * c["Hkv"] * c["nq"]
        live = tokens * (share if 2 * c["nq"] > c["nk"] else 1.0)
        # in to the cache, back out of it; places without a token come back as zeros
        return {"bytes": 2 * c["d"] * elem * (live + tokens) + 2 * live * held, "flops": 8 * live * c["d"]}
    tokens = c["B"] * c["Hkv"] * c["nk"]
    if c["op"] == "read":
        return {"bytes": tokens * share * held + 2 * tokens * c["d"] * elem, "flops": 2 * tokens * share * c["d"]}
    return {"bytes": tokens * share * held + 2 * c["B"] * c["H"] * c["nq"] * c["d"] * elem,
            "flops": 4 * _pairs(c) * c["d"]}


def _held(x):
    """What the cache holds of x, in float64: in a block of 32 of step s the nearest multiple of s/2 up to 2 s, of
    s up to 4 s, of 2 s beyond, at most 6 s, ties to the even multiple."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 7.0))
    e = torch.where(top > 7 * torch.exp2(e), e + 1, e)                   # log2 rounded past a whole number
    e = torch.where(top <= 7 * torch.exp2(e - 1), e - 1, e)
    e = torch.where(top > 0, e, -125.0).clamp(-125, 125)
    y = x / torch.exp2(e)
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return (y.sign() * (torch.round(a / step) * step).clamp(max=6.0) * torch.exp2(e)).flatten(-2)


def exact(case, seed):
    c = case
    if c["op"] == "rotary":
        return _exact_rotary(c, _rotary_inputs(c, seed))
    s = _cache_inputs(c, seed)
    k, v, n, lengths = s["k"], s["v"], s["n"], s["lengths"]
    if c["op"] != "attend":
        counts = lengths if s["counts"] is None else s["counts"]
        live = (torch.arange(n, device="cuda") < counts[:, None])[:, None, :, None]
        return tuple(torch.where(live, _held(x), 0.0) for x in (k, v))
    B, H, nq, nk, d = (c[x] for x in ("B", "H", "nq", "nk", "d"))
    group = H // c["Hkv"]
    out = torch.zeros(B, H, nq, d, dtype=torch.float64, device="cuda")
    for b in range(B):
        m = int(lengths[b])
        for h in range(c["Hkv"]):
            K, V = _held(k[b, h, :m]), _held(v[b, h, :m])
            for g in range(h * group, (h + 1) * group):
                logits = s["q"][b, g].double() @ K.t() / math.sqrt(d)
                if c["causal"]:
                    later = torch.arange(m, device="cuda") > (m - nq + torch.arange(nq, device="cuda"))[:, None]
                    logits = logits.masked_fill(later, -math.inf)
                out[b, g] = torch.softmax(logits, -1) @ V
    return out


def _exact_rotary(c, s):
    """Rotation as a product of complex numbers, gradients by autograd."""
    r, half = c["rot"], c["pairs"] == "half"
    turn = torch.polar(torch.full((), _magnitude(c), dtype=torch.float64, device="cuda"),
                       s["positions"].double()[:, None, :, None] * _frequencies(c).to("cuda"))
    train = c["mode"] == "train"
    x = [s[n].detach().double().requires_grad_(train) for n in ("q", "k")]
    w = [s[n].detach().double().requires_grad_(train) for n in ("wq", "wk") if s[n] is not None]
    results = []
    with torch.set_grad_enabled(train):
        for i, t in enumerate(x):
            if w:
                t = t / torch.sqrt(t.square().mean(-1, keepdim=True) + EPS) * w[i]
            pair = torch.stack((t[..., : r // 2], t[..., r // 2: r]), -1) if half else t[..., :r].unflatten(-1, (-1, 2))
            z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
            z = torch.cat((z[..., 0], z[..., 1]), -1) if half else z.flatten(-2)
            results.append(torch.cat((z, t[..., r:]), -1))
    if not train:
        return tuple(results)
    grads = torch.autograd.grad(results, x + w, (s["gq"].double(), s["gk"].double()))
    return (*(t.detach() for t in results), *grads)
