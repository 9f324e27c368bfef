"""Normed and turned heads by their definition in 64 bits, and the error that fp32 arithmetic and one rounding allow.

Counted in roundings of fp32, e = 2^-24: the sum of D squares is 8 multiply-adds in a lane, 4 additions of lanes and one of eps,
half of which the root leaves (6.5 e), the reciprocal root itself 2 e; x r w another 2 e; a cosine or sine 4 e (its argument, up to
pi / 4, goes through three roundings, 2 e; the series ends below e / 8; two roundings near 1); the multiply-add of a pair 1 e.  16 e = 2^-20 of the
magnitudes of both values of a pair covers a forward value.  Angles: positions times frequencies in doubles, three roundings
of 2^-53 here and there: 2^-51 of the angle.
"""
import torch

from tests.attn_util import half_step, least

E = 2.0 ** -24


def angles(positions, freq, axis, B, S):
    """[B, S, pairs] in 64 bits from positions [S], [B, S] or [axes, B, S]."""
    p = positions if positions.dim() == 3 else positions.expand(B, S)[None]
    which = torch.zeros(freq.shape[0], dtype=torch.long, device=freq.device) if axis is None else axis.long()
    there = which < p.shape[0]
    theta = p[which.clamp(max=p.shape[0] - 1)].permute(1, 2, 0).double() * freq.double()
    return torch.where(there, theta, 0.0)


def pair_up(x, pairs, adjacent):
    """The two values of each pair of x [.., D], and what is in none."""
    if adjacent:
        return x[..., 0 : 2 * pairs : 2], x[..., 1 : 2 * pairs : 2], x[..., 2 * pairs:]
    return x[..., :pairs], x[..., pairs : 2 * pairs], x[..., 2 * pairs:]


def put_back(a, b, rest, adjacent):
    turned = torch.stack([a, b], -1).flatten(-2) if adjacent else torch.cat([a, b], -1)
    return torch.cat([turned, rest], -1)


def turn(x, theta, adjacent):
    """x [B, H, S, D] turned by theta [B, S, pairs]."""
    if theta is None:
        return x
    a, b, rest = pair_up(x, theta.shape[-1], adjacent)
    c, s = torch.cos(theta)[:, None], torch.sin(theta)[:, None]
    return put_back(a * c - b * s, a * s + b * c, rest, adjacent)


def both(x, theta, adjacent):
    """Of each value the magnitude of it and its partner together, and what an error of the angle may make of it."""
    if theta is None:
        return x.abs(), torch.zeros_like(x)
    a, b, rest = pair_up(x.abs(), theta.shape[-1], adjacent)
    off = 2.0 ** -51 * theta.abs()[:, None] * (a + b)
    return put_back(a + b, a + b, rest, adjacent), put_back(off, off, torch.zeros_like(rest), adjacent)


def forward(x, weight, eps, theta, adjacent):
    """y in 64 bits and the error allowed."""
    dtype, x = x.dtype, x.double()
    u = x
    if weight is not None:
        u = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * weight.double()
    y = turn(u, theta, adjacent)
    size, off = both(u, theta, adjacent)
    return y, half_step(dtype) * y.abs() + 2.0 ** -20 * size + off + least(dtype)


def gradient(x, weight, eps, theta, adjacent, dy):
    """dx and its allowed error, dw and its own.  With G = (|dy_e| + |dy_p|) w: g w is off by 8 e of G, n by 10 e, mean(g w n) by 8 + 10
    + 13 e of the mean of G |n|, its product with n by another 11, r by 9: 64 e = 2^-18 of r (G + |n| mean(G |n|)) covers dx.
    A sum of dw's terms (20 e each) goes through a thread's rows, at most 256 here, and three short sums of 32: 384 e."""
    dtype = dy.dtype
    dy = dy.double()
    g = turn(dy, None if theta is None else -theta, adjacent)
    size, off = both(dy, theta, adjacent)
    if weight is None:
        return g, half_step(dtype) * g.abs() + 8 * E * size + off + least(dtype), None, None
    x, w = x.double(), weight.double()
    r = 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    n = x * r
    dx = r * (g * w - n * (g * w * n).mean(-1, keepdim=True))
    G = (size * 64 * E + off) * w.abs()
    tx = half_step(dtype) * dx.abs() + r * (G + n.abs() * (G * n.abs()).mean(-1, keepdim=True)) + least(dtype)
    dims = tuple(range(x.dim() - 1))
    return dx, tx, (g * n).sum(dims), ((384 * E * size + off) * n.abs()).sum(dims)
