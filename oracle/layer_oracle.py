"""Rotary positions, head norms and the 4-bit cache's rounding in float64 (plain torch,
any device), written from the definitions of mra_layer.h: the oracle of their tests."""
import torch

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
# 2 pi = TURN[0] + TURN[1] + TURN[2], the first of 23 bits: exact times a number of turns below 2^30
TURN = (float.fromhex("0x1.921fb4p+2"), float.fromhex("0x1.4442d18469899p-22"), float.fromhex("-0x1.9d747f23e32edp-77"))


def angles(n, freqs, positions, magnitude=1.0):
    """cos and sin times the magnitude, [B or 1, 1, n, r / 2]. Positions have 32 bits, so their product with a
    frequency's first 21 bits is exact; whole turns leave it before the rest comes in, and the angle is
    off by less than 2^-40 at every position (a float64 product: by 2^-23 at 2^31)."""
    p = torch.arange(n, device=freqs.device) if positions is None else positions
    p, f = (p if p.dim() == 2 else p[None]).double()[:, None, :, None], freqs.double()
    c = f * (2.0 ** 32 + 1)
    first = c - (c - f)
    t = p * first
    k = torch.round(t / (TURN[0] + TURN[1]))
    t = ((t - k * TURN[0]) - k * TURN[1]) - k * TURN[2] + p * (f - first)
    return torch.cos(t) * magnitude, torch.sin(t) * magnitude


def pairs(x, r, interleaved):
    return (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., : r // 2], x[..., r // 2: r])


def unpair(a, b, x, interleaved):
    r = 2 * a.shape[-1]
    y = torch.stack((a, b), -1).flatten(-2) if interleaved else torch.cat((a, b), -1)
    return torch.cat((y, x[..., r:]), -1)


def turn(x, freqs, positions=None, interleaved=False, magnitude=1.0, back=False, absolute=False):
    """x turned (``back``: by the opposite angles); ``absolute``: the sum of the terms' largest magnitudes."""
    x = x.double()
    if freqs is None or not len(freqs):
        return x.abs() if absolute else x
    c, s = angles(x.shape[2], freqs, positions, magnitude)
    a, b = pairs(x, 2 * len(freqs), interleaved)
    if absolute:
        m = abs(magnitude) * (a.abs() + b.abs())
        return unpair(m, m, x.abs(), interleaved)
    s = -s if back else s
    return unpair(a * c - b * s, b * c + a * s, x, interleaved)


def normed(x, eps):
    x = x.double()
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    return x * r, r


def rotary(x, freqs, weight=None, eps=1e-6, absolute=False, **kw):
    y = x.double()
    if weight is not None:
        y = normed(x, eps)[0] * weight.double()
    return turn(y, freqs, absolute=absolute, **kw)


def rotary_grads(g, x, freqs, weight=None, eps=1e-6, absolute=False, **kw):
    """(dx, dw) by the chain rule; ``absolute``: the sums over the magnitudes of their terms."""
    g = turn(g, freqs, back=True, absolute=absolute, **kw)
    if weight is None:
        return g, None
    y, r = normed(x, eps)
    w = weight.double()
    if absolute:
        y, w = y.abs(), w.abs()
    h = g * w
    m = (h * y).mean(-1, keepdim=True)
    return r * (h + y * m if absolute else h - y * m), (g * y).sum((0, 1, 2))


def held(x):
    """What the cache holds of x [..., d], and the exponents [..., d / 32]."""
    x = x.double().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, 125.0)
    for k in range(124, -126, -1):                       # the smallest power of two with top <= 7 of it
        e = torch.where(top <= 7.0 * 2.0 ** k, float(k), e)
    y = x / torch.exp2(e)
    dist = (y.abs().unsqueeze(-1) - torch.tensor(GRID, dtype=torch.float64, device=x.device)).abs()
    near = dist.amin(-1, keepdim=True)
    code = torch.arange(8, device=x.device)
    ties = dist == near                                  # two of them: the even code
    code = torch.where(ties & ((code % 2 == 0) | (ties.sum(-1, keepdim=True) == 1)), code, -1).amax(-1)
    v = torch.tensor(GRID, dtype=torch.float64, device=x.device)[code] * torch.where(y < 0, -1.0, 1.0)
    return (v * torch.exp2(e)).flatten(-2), e.squeeze(-1).long()


def page_bytes(k, v):
    """The bytes of one page of one head, of its tokens' k and v [page_size, d] (host tensors)."""
    codes, steps = [], []
    for x in (k, v):
        h, e = held(x)
        y = (h.unflatten(-1, (-1, 32)) / torch.exp2(e.double())[..., None]).flatten(-2)
        c = (y.abs().unsqueeze(-1) == torch.tensor(GRID, dtype=torch.float64)).int().argmax(-1) + 8 * (y < 0).int()
        codes.append(c[:, 0::2] | c[:, 1::2] << 4)
        steps.append(e + 127)
    return torch.cat([p.flatten().to(torch.uint8) for p in codes + steps])
