"""The attention operators' definitions in 64 bits, and the error that their types allow, term by term.

u is half a step of the type (a rounding to it is off by at most u relative to the value).  The kernels round the
probabilities (and, in the gradient, dS) to the type once and the result once; everything else is fp32, whose share
(scores of a few tens in the exponent, sums of a few thousand terms) stays below F = 2^-14 of the sums of magnitudes.
"""
import math

import torch

F = 2.0 ** -14


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def least(dtype):
    """Half the distance of the type's smallest values: what rounding to it costs below its normal range."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def visible(n_q, n_k, window, sinks, device="cpu"):
    p = torch.arange(n_k - n_q, n_k, device=device)[:, None]
    j = torch.arange(n_k, device=device)[None]
    see = j <= p
    if window:
        see &= ((p - j) < window) | (j < sinks)
    return see


def forward(q, k, v, window, sinks, scale):
    """q [B, Hq, Sq, D], k, v [B, Hkv, Sk, D]: P [B, Hq, Sq, Sk], o, lse in 64 bits; masked places do not enter."""
    q, k, v = q.double(), k.double(), v.double()
    group = q.shape[1] // k.shape[1]
    k, v = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    see = visible(q.shape[2], k.shape[2], window, sinks, q.device)
    s = torch.matmul(q, k.transpose(2, 3)) * scale
    s = s.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    return p, torch.matmul(p, v), lse


def o_bound(p, v, dtype):
    group = p.shape[1] // v.shape[1]
    return (2 * half_step(dtype) + F) * torch.matmul(p, v.double().abs().repeat_interleave(group, 1)) + least(dtype)


def gradients(q, k, v, d_o, window, sinks, scale, dtype):
    """dq, dk, dv in 64 bits and the errors that each is allowed."""
    p, o, _ = forward(q, k, v, window, sinks, scale)
    b, hq, n_q, d = q.shape
    hkv, n_k = k.shape[1:3]
    u = half_step(dtype)
    q, k, v, d_o = q.double(), k.double(), v.double(), d_o.double()
    kk, vv = k.repeat_interleave(hq // hkv, 1), v.repeat_interleave(hq // hkv, 1)
    dp = torch.matmul(d_o, vv.transpose(2, 3))
    ds = p * (dp - (d_o * o).sum(-1, keepdim=True))
    # dS is rounded once (u), stands on P and dP in fp32 (F), and on delta, from an o that may be o_bound off
    pv = torch.matmul(p, vv.abs())
    off = (u + F) * ds.abs() + p * (F * torch.matmul(d_o.abs(), vv.abs().transpose(2, 3)) + (2 * u + F) * (d_o.abs() * pv).sum(-1, keepdim=True))
    fold = lambda x: x.view(b, hkv, hq // hkv, n_k, d).sum(2)  # noqa: E731
    dq, dk, dv = torch.matmul(ds, kk) * scale, fold(torch.matmul(ds.transpose(2, 3), q)) * scale, fold(torch.matmul(p.transpose(2, 3), d_o))
    tq = torch.matmul(off, kk.abs()) * scale + u * dq.abs()
    tk = fold(torch.matmul(off.transpose(2, 3), q.abs())) * scale + u * dk.abs()
    tv = (2 * u + F) * fold(torch.matmul(p.transpose(2, 3), d_o.abs()))
    return tuple((x, t + least(dtype)) for x, t in ((dq, tq), (dk, tk), (dv, tv)))


def assert_within(got, want, bound, what=""):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), (what, "NaN in other places")
    off = (got - want).abs() - bound
    off = off[~torch.isnan(off)]
    assert off.numel() == 0 or float(off.max()) <= 0, (what, float(off.max()), float((off > 0).double().mean()))


def assert_lse(got, want):
    empty = want == -math.inf
    assert torch.equal(got == -math.inf, empty)
    assert bool(((got.double() - want)[~empty].abs() <= F * (1 + want[~empty].abs())).all())


def quantise(x, dtype):
    """Rows of x [..., D] as a cache holds them: e4m3 code values, exponent byte, in 64 bits by the definition."""
    x = x.double().cpu()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), 0.0).amax(-1)
    e = torch.zeros_like(top, dtype=torch.long)
    for at in range(-126, 129):  # the least e with top <= 448 2^e
        e = torch.where((top > 448.0 * 2.0 ** (at - 1)) | (at == -126), torch.tensor(at), e)
    e = torch.where(top == 0, 0, e)
    y = torch.ldexp(x, -e[..., None].double())
    _, x2 = torch.frexp(torch.where(finite, y, 1.0))
    grain = torch.ldexp(torch.ones_like(y), (x2 - 4).clamp(min=-9).double())
    code = torch.where(finite, torch.round(y / grain) * grain, math.nan)
    return code, e + 127
