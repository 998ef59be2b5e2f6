"""Exact softmax attention, its gradients and its position bias in float64 (plain
torch, any device), written from the definition: the oracle of the tests."""
import math

import torch


def logits(q, k, scale, causal=False, lengths=None, key_mask=None, q_start=None, bias=None, buckets=None):
    """S [B, H, nq, nk] in float64 and which entries count."""
    B, H, nq, d = q.shape
    nk, group = k.shape[2], H // max(k.shape[1], 1)
    K = k.double().repeat_interleave(group, 1)
    S = q.double() @ K.transpose(2, 3).contiguous() * (d ** -0.5 if scale is None else scale)
    key = torch.arange(nk, device=q.device)
    start = torch.full((B,), nk - nq, device=q.device) if q_start is None else q_start.long()
    pos = start[:, None] + torch.arange(nq, device=q.device)
    rel = key - pos[:, :, None]                                   # [B, nq, nk]
    if bias is not None:
        far = buckets.numel() // 2
        at = buckets.long()[rel.clamp(-far, far) + far]
        known = (at >= 0) & (at < bias.shape[0])
        t = bias.double()[at.clamp(0, bias.shape[0] - 1)]         # [B, nq, nk, H]
        S = S + torch.where(known[..., None], t, 0.0).permute(0, 3, 1, 2)
    keep = torch.ones(B, 1, nk, dtype=torch.bool, device=q.device)
    if lengths is not None:
        keep = keep & (key < lengths[:, None, None])
    if key_mask is not None:
        keep = keep & key_mask[:, None].bool()
    keep = keep.expand(B, nq, nk)
    if causal:
        keep = keep & (rel <= 0)
    return S, keep[:, None]


def _clean(x, lengths, key_mask):
    """Rows that count for no query as zeros (they may hold anything)."""
    B, _, nk, _ = x.shape
    keep = torch.ones(B, nk, dtype=torch.bool, device=x.device)
    if lengths is not None:
        keep &= torch.arange(nk, device=x.device) < lengths[:, None]
    if key_mask is not None:
        keep &= key_mask.bool()
    return torch.where(keep[:, None, :, None], x.double(), 0.0)


def attention(q, k, v, scale=None, lengths=None, key_mask=None, **kw):
    """(Z, L, P), float64."""
    k, v = _clean(k, lengths, key_mask), _clean(v, lengths, key_mask)
    S, keep = logits(q, k, scale, lengths=lengths, key_mask=key_mask, **kw)
    S = S.masked_fill(~keep, -math.inf)
    L = torch.logsumexp(S, -1) if S.shape[-1] else S.new_full(S.shape[:3], -math.inf)
    P = torch.exp(S - torch.where(L == -math.inf, 0.0, L)[..., None])
    V = v.repeat_interleave(q.shape[1] // max(k.shape[1], 1), 1)
    return P @ V, L, P


def gradients(q, k, v, g, scale=None, lengths=None, key_mask=None, absolute=False, **kw):
    """(dq, dk, dv, dbias) by the chain rule; ``absolute``: the sums over the
    magnitudes of their terms (delta's included), which bound what roundings of
    the terms can move the gradients by."""
    B, H, nq, d = q.shape
    Hkv, nk = k.shape[1:3]
    group = H // max(Hkv, 1)
    Z, _, P = attention(q, k, v, scale, lengths, key_mask, **kw)
    f = torch.abs if absolute else (lambda x: x)
    K, V = (f(_clean(x, lengths, key_mask)).repeat_interleave(group, 1) for x in (k, v))
    Q, G = f(q.double()), f(g.double())
    dP = G @ V.transpose(2, 3).contiguous()
    delta = (G * (P @ V if absolute else Z)).sum(-1, keepdim=True)
    dS = P * (dP + delta if absolute else dP - delta)
    c = d ** -0.5 if scale is None else scale
    dq = c * (dS @ K)
    dk = c * (dS.transpose(2, 3).contiguous() @ Q)
    dv = P.transpose(2, 3).contiguous() @ G
    dk, dv = (x.view(B, Hkv, group, nk, d).sum(2) if H else x for x in (dk, dv))
    db = None
    if kw.get("bias") is not None:
        bias, buckets, start = kw["bias"], kw["buckets"], kw.get("q_start")
        far = buckets.numel() // 2
        start = torch.full((B,), nk - nq, device=q.device) if start is None else start.long()
        pos = start[:, None] + torch.arange(nq, device=q.device)
        rel = torch.arange(nk, device=q.device) - pos[:, :, None]
        at = buckets.long()[rel.clamp(-far, far) + far]
        db = torch.stack([(dS * (at == c)[:, None]).sum((0, 2, 3)) for c in range(bias.shape[0])])
    return dq, dk, dv, db
