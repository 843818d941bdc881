"""Plain fp64 definitions of the cache operators (rotary positions, 8-bit rows, tree
attention), on CPU tensors; test infrastructure only."""
from __future__ import annotations

import math

import torch


def frequencies(dim, base=10000.0, scaling="none", factor=1.0, original=0.0, fast=32.0, slow=1.0):
    """(theta [dim / 2] in fp64, factor on the rotated values)."""
    if scaling == "ntk":
        base = base * factor ** (dim / (dim - 2.0))
    theta = torch.tensor([base ** (-2.0 * p / dim) for p in range(dim // 2)], dtype=torch.float64)
    if scaling == "linear":
        theta = theta / factor
    if scaling == "yarn":
        mix = [min(1.0, max(0.0, (original * float(t) / (2 * math.pi) - slow) / (fast - slow))) for t in theta]
        g = torch.tensor(mix, dtype=torch.float64)
        return (1 - g) * theta / factor + g * theta, 0.1 * math.log(factor) + 1.0
    return theta, 1.0


def rotate(x, positions, theta, scale=1.0, layout="half", transpose=False):
    """x [rows, heads, hd] in fp64, pairs of the first 2 len(theta) values turned."""
    y = x.double().clone()
    half = len(theta)
    for p in range(half):
        i, j = (p, p + half) if layout == "half" else (2 * p, 2 * p + 1)
        ang = positions.double() * theta[p] * (-1.0 if transpose else 1.0)
        c, s = (scale * torch.cos(ang))[:, None], (scale * torch.sin(ang))[:, None]
        a, b = x[..., i].double(), x[..., j].double()
        y[..., i], y[..., j] = a * c - b * s, b * c + a * s
    return y


def e4m3_values():
    """The non-negative finite E4M3 values in order."""
    v = [m * 2.0 ** -9 for m in range(8)]
    v += [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8) if not (e == 15 and m == 7)]
    return torch.tensor(v, dtype=torch.float64)


def quantise(x):
    """Rows [.., hd] in fp64: (what is stored [.., hd], exponent bytes [..]); NaN for what is not finite."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x, 0.0).abs().amax(-1)
    e = torch.full(top.shape, -126, dtype=torch.int64)
    for idx in torch.nonzero(top > 0):
        i, t = tuple(idx.tolist()), float(top[tuple(idx.tolist())])
        n = -126
        while t > 448.0 * 2.0 ** n:
            n += 1
        e[i] = n
    grid = e4m3_values()
    u = torch.where(finite, x, 0.0) / torch.exp2(e.double())[..., None]
    a = u.abs()
    hi = torch.searchsorted(grid, a.contiguous()).clamp_max(len(grid) - 1)
    lo = (hi - 1).clamp_min(0)
    dh, dl = grid[hi] - a, a - grid[lo]
    even_hi = hi % 2 == 0  # the list index is the bit pattern
    pick = torch.where((dh < dl) | ((dh == dl) & even_hi), hi, lo)
    v = torch.copysign(grid[pick], u)
    return torch.where(finite, v, math.nan), (e + 127)


def tree_attention(q, kc, vc, k, v, see, scale=None):
    """One sequence.  q [T, nq, hd]; kc, vc [nkv, N, hd] cached; k, v [T, nkv, hd]; see [T, T] bool.
    Returns (out [T, nq, hd], lse [T, nq], weight of |v| [T, nq, hd], largest sum |q||k| scale)."""
    t, nq, hd = q.shape
    nkv = k.shape[1]
    group = nq // nkv
    scale = hd ** -0.5 if scale is None else scale
    out = torch.zeros((t, nq, hd), dtype=torch.float64)
    mag = torch.zeros_like(out)
    lse = torch.full((t, nq), -math.inf, dtype=torch.float64)
    big = 0.0
    for i in range(t):
        cols = [j for j in range(t) if see[i, j]]
        for h in range(nq):
            g = h // group
            kk = torch.cat([kc[g].double(), k[cols, g].double()])
            vv = torch.cat([vc[g].double(), v[cols, g].double()])
            if kk.shape[0] == 0:
                continue
            s = (kk @ q[i, h].double()) * scale
            big = max(big, float((kk.abs() @ q[i, h].double().abs()).nan_to_num(0.0, 0.0).max()) * scale)
            m = s.max()
            p = torch.exp(s - m)
            l = p.sum()
            lse[i, h] = m + torch.log(l)
            out[i, h] = (p / l) @ vv
            mag[i, h] = (p / l) @ vv.abs()
    return out, lse, mag, big
