"""Plain definitions, in 64 bits, of a cache held in four bits, of phase 2 over it, and of queries and keys that are normed and
rotated; written from include/star_attn.h's text and sharing no code with the package."""
import math

import torch

GRID = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)
# (a device's power function need not be exact at whole numbers: Python's are)
UNIT = torch.tensor([2.0 ** (e - 127) for e in range(255)] + [math.nan], dtype=torch.float64)


def quantise(x):
    """x [..., d] -> codes [..., d / 2] and exponents [..., d / 32], uint8.  A search over the grid, not arithmetic on bits."""
    g = x.double().unflatten(-1, (-1, 32))
    most = g.abs().amax(-1)
    fine = torch.isfinite(g).all(-1)
    e = torch.full_like(most, 2)
    e[fine] = (torch.floor(torch.log2((most[fine] / 3.5).clamp(min=2.0 ** -200))) + 127).clamp(2, 252)
    # (log2 may be off by a last bit next to a power of two)
    unit = UNIT.to(x.device)
    for _ in range(2):
        up = fine & (e < 252) & (3.5 * unit[(e + 1).long()] <= most)
        down = fine & (e > 2) & (3.5 * unit[e.long()] > most)
        e = e + up.double() - down.double()
    e[fine & (most == 0)] = 127
    y = g.abs() / unit[e.long()][..., None]
    y = torch.where(fine[..., None], y, torch.zeros_like(y))
    off = (y[..., None] - GRID.to(x.device)).abs()
    best = off.amin(-1, keepdim=True)
    near = off == best
    odd = torch.arange(8, device=x.device) % 2 == 1
    both = near.sum(-1, keepdim=True) > 1
    code = (near & ~(both & odd)).to(torch.int64).argmax(-1)
    code = code + 8 * torch.signbit(g).to(torch.int64)
    code[~fine] = 0
    e[~fine] = 255
    code = code.flatten(-2)
    return (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8), e.to(torch.uint8)


def values(codes, exponents):
    """What they stand for, float64."""
    c = codes.to(torch.int64)
    c = torch.stack([c % 16, c // 16], -1).flatten(-2)
    x = GRID.to(codes.device)[c % 8] * torch.where(c >= 8, -1.0, 1.0)
    unit = UNIT.to(codes.device)[exponents.long()]
    return (x.unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)


def attend(Q, K, V, scale, cache_len=None, lo=0, hi=None):
    """Q [q, d] of one head against rows [lo, hi) of K, V [n, d], new token j seeing rows up to cache_len + j (None: all).
    Returns A [q, d], lse [q], and what error bounds are made of: sum p |v| [q, d], the largest sum |q k| scale of a row [q], and
    the sum of |v| over the seen keys whose values fp16 holds [q, d]."""
    Q, K, V = Q.double(), K.double(), V.double()
    hi = K.shape[0] if hi is None else hi
    seen = torch.zeros(Q.shape[0], K.shape[0], dtype=torch.bool, device=Q.device)
    for j in range(Q.shape[0]):
        end = hi if cache_len is None else min(hi, cache_len + j + 1)
        seen[j, lo:max(lo, end)] = True
    s = torch.where(seen, Q @ K.T * scale, torch.tensor(-math.inf, dtype=torch.float64, device=Q.device))
    lse = torch.logsumexp(s, -1)
    p = torch.where(seen, torch.exp(s - lse[:, None]), torch.zeros_like(s))
    pick = lambda X: torch.stack([p[j, r] @ X[r] for j, r in enumerate(seen)])
    if torch.isfinite(V).all():
        pick = lambda X: p @ X
    size = torch.where(seen, Q.abs() @ K.abs().T * scale, torch.zeros_like(s)).amax(-1)
    held = torch.where(V.abs() <= 6 * 2.0 ** 13, V.abs(), torch.zeros_like(V))
    return pick(V), lse, pick(V.abs()), size, seen.double() @ held


def norm_rope(x, weight, eps, theta, positions, axis):
    """x [B, T, H, d]; positions [B, T, n] (integers); axis: of each of the d / 2 frequencies.  weight None: not normed.
    Returns the result and, for bounds, |n_i| + |n_(i + d/2)| of every pair, [B, T, H, d / 2]."""
    x = x.double()
    d = x.shape[-1]
    if weight is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * weight.double()
    freq = torch.tensor([float(theta) ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=x.device)
    ang = positions.double()[..., torch.as_tensor(axis, device=x.device)] * freq
    c, s = torch.cos(ang)[:, :, None], torch.sin(ang)[:, :, None]
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return torch.cat([lo * c - hi * s, hi * c + lo * s], -1), lo.abs() + hi.abs()
