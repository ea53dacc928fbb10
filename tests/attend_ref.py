"""Attention over the bank and its gradients in 64 bits, with bounds for a
32-bit computation of them, and 4-bit rows by table (plain torch, any device).

Bounds. With u = 2^-24, a score's half distance a = <q,x> - |q|^2/2 - |x|^2/2 is a
sum of d + 2 terms whose partial sums stay under S = |q||x| + |q|^2/2 + |x|^2/2.
Their roundings, each at most u*S, are independent, so a is off by a few times
sqrt(d + 2) * u * S; the bound takes four times that, plus 4*u*S for the norms'
own. A weight exp(2*beta*a - lse) is then off by a factor within
  E = 2*beta*|da| + 8*u*(1 + 2*beta*|a - lse/(2*beta)|),
the second part for the multiply-add, the power of two and lse as it is stored.
A weight, or a product with one, that falls under T = 2^-126, the least normal
32-bit number, may be taken as 0: that is off by T at most. (At beta = 50 rows
two apart have weights of e^-100 = 4e-44; products with them leave the range
long before the weights' sums do.)
"""
import math

import torch

U = 2.0 ** -24
T = 2.0 ** -126
MAGNITUDES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def unpack4(rows, scales):
    """Values (float64) of rows held in 4 bits."""
    N, half = rows.shape
    table = torch.tensor(MAGNITUDES + [-m for m in MAGNITUDES], dtype=torch.float64,
                         device=rows.device)
    r = rows.long()
    v = torch.stack((table[r % 16], table[r // 16]), 2).reshape(N, half // 16, 32)
    return (v * 2.0 ** (scales.double() - 127.0)[..., None]).reshape(N, 2 * half)


def weights(q, x, beta, mask, lse=None):
    """(p, E, lse, dist, live) in 64 bits; rows whose mask is 0 are taken as zeros."""
    q = q.double()
    live = torch.ones(x.shape[0], dtype=torch.bool, device=x.device) if mask is None else mask != 0
    x = torch.where(live[:, None], x.double(), torch.zeros_like(x, dtype=torch.float64))
    d = q.shape[1]
    q2, x2 = (q * q).sum(1)[:, None], (x * x).sum(1)[None]
    dist = q2 + x2 - 2.0 * q @ x.t()
    # (the expanded form in 64 bits is good to 2^-50 of the norms)
    score = torch.where(live[None], -beta * dist, torch.full_like(dist, -math.inf))
    if lse is None:
        lse = torch.logsumexp(score, 1)
    lse = lse.double()
    dead = torch.isneginf(lse)
    safe = torch.where(dead, torch.zeros_like(lse), lse)
    p = torch.where(dead[:, None], torch.zeros_like(score), torch.exp(score - safe[:, None]))
    S = torch.sqrt(q2 * x2) + 0.5 * q2 + 0.5 * x2
    da = (4.0 * math.sqrt(d + 2) + 4.0) * U * S
    arg = torch.where(torch.isinf(score), torch.zeros_like(score), score - safe[:, None])
    E = 2.0 * beta * da + 8.0 * U * (1.0 + arg.abs() + beta * dist.abs() + safe.abs()[:, None])
    return p, E, lse, dist, live, x


def attend(q, x, beta, qual, length, mask=None):
    """{name: (value, bound)} of the forward pass."""
    p, E, lse, dist, live, _ = weights(q, x, beta, mask)
    v = torch.cat((qual, length), 1).double()
    v = torch.where(live[:, None], v, torch.zeros_like(v))
    M = qual.shape[1]
    dead = torch.isneginf(lse)[:, None]
    nan = torch.full((q.shape[0], 2 * M), math.nan, dtype=torch.float64, device=q.device)
    out = torch.where(dead, nan, p @ v)
    # weights off by E each, the sums by a few roundings of their partial sums
    n = math.sqrt(x.shape[0]) + 16.0
    e = (p * E).sum(1, keepdim=True)
    bound = (p * E) @ v.abs() + (e + n * U) * (p @ v.abs()) + T * (v.abs().sum(0) + x.shape[0])
    lb = (p * E).sum(1) + n * U + 4.0 * U * lse.abs()
    return {"q_hat": (out[:, :M], bound[:, :M]), "l_hat": (out[:, M:], bound[:, M:]),
            "lse": (lse, lb)}


def usage(q, x, beta, lse, old, decay, mask=None):
    p, E, _, _, _, _ = weights(q, x, beta, mask, lse)
    s = p.sum(0)
    return (decay * old.double() + s,
            (p * E).sum(0) + (math.sqrt(q.shape[0]) + 4.0) * U * (s + old.double().abs()) +
            q.shape[0] * T)


def backward(q, x, beta, qual, length, q_hat, l_hat, lse, dq_hat, dl_hat, dlse=None, mask=None):
    """{name: (value, bound)} of the gradients; bounds before the outputs' own rounding."""
    bf16 = q.dtype == torch.bfloat16
    p, E, _, dist, live, x = weights(q, x, beta, mask, lse)
    q = q.double()
    dead = torch.isneginf(lse)[:, None]
    v = torch.cat((qual, length), 1).double()
    v = torch.where(live[:, None], v, torch.zeros_like(v))
    zero = torch.zeros(q.shape[0], v.shape[1], dtype=torch.float64, device=q.device)
    do = torch.where(dead, zero, torch.cat((dq_hat, dl_hat), 1).double())
    o = torch.where(dead, zero, torch.cat((q_hat, l_hat), 1).double())
    M = qual.shape[1]
    shift = (do * o).sum(1, keepdim=True)
    size = do.abs() @ v.abs().t() + (do * o).abs().sum(1, keepdim=True)
    if dlse is not None:
        dl = torch.where(dead, zero[:, :1], dlse.double()[:, None])
        shift = shift - dl
        size = size + dl.abs()
    g = p * (do @ v.t() - shift)
    # p, the 2M + 2 terms of the weights' gradient, and two bf16 values: off by
    # half a step of the second (2^-9 * 2^-9) at most
    eg = g.abs() * (E + 2 * U + (2.0 ** -18 if bf16 else 0.0)) + p * (2 * M + 6) * U * size + \
        2 * T * (1.0 + size)
    # sums over n terms, and the difference of two of them
    def summed(ga, ea, y, own, n):
        """bound of 2 beta (ga @ y - sum(ga) * own)"""
        far = (math.sqrt(n) + 16.0) * U
        return 2.0 * beta * (ea @ y.abs() + ea.sum(1, keepdim=True) * own.abs() +
                             far * (ga.abs() @ y.abs() +
                                    ga.abs().sum(1, keepdim=True) * own.abs()) + n * T)
    eq = summed(g, eg, x, q, x.shape[0])
    ex = summed(g.t(), eg.t(), q, x, q.shape[0])
    dq = 2.0 * beta * (g @ x - g.sum(1, keepdim=True) * q)
    dx = 2.0 * beta * (g.t() @ q - g.sum(0)[:, None] * x)
    dv = p.t() @ do
    ev = (p * E).t() @ do.abs() + (math.sqrt(q.shape[0]) + 8.0) * U * (p.t() @ do.abs()) + \
        T * (do.abs().sum(0) + q.shape[0])
    edist = 2.0 * (4.0 * math.sqrt(q.shape[1] + 2) + 4.0) * U * (
        (q * q).sum(1)[:, None] + (x * x).sum(1)[None])
    db = -(g * dist).sum(1)
    eb = (eg * dist.abs() + g.abs() * edist).sum(1) + \
        (math.sqrt(x.shape[0]) + 16.0) * U * (g.abs() * dist.abs()).sum(1)
    return {"d_queries": (dq, eq), "d_bank": (dx, ex), "d_qual": (dv[:, :M], ev[:, :M]),
            "d_len": (dv[:, M:], ev[:, M:]), "d_beta": (db, eb)}


def check(name, got, value, bound, label=""):
    """got is within bound of value, plus half a step of its type; NaN and inf where
    value has them. Returns the largest share of the bound that is used."""
    got = got.double()
    bad = ~torch.isfinite(value)
    assert torch.equal(torch.isnan(got), torch.isnan(value)), f"{label} {name}: NaN elsewhere"
    assert torch.equal(got[bad & ~torch.isnan(value)], value[bad & ~torch.isnan(value)]), \
        f"{label} {name}: infinities elsewhere"
    err = torch.where(bad, torch.zeros_like(value), (got - value).abs())
    share = torch.where(bad, torch.zeros_like(value), err / bound)
    worst = float(share.max()) if share.numel() else 0.0
    assert worst <= 1.0, f"{label} {name}: {worst:.2f} times the bound, " \
        f"largest error {float(err.max()):.3g} of {float(value[~bad].abs().max()):.3g}"
    return worst
