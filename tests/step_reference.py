"""The operators around the linears from their definitions, in 64 bits on the CPU
(plain torch; shares nothing with the package), and bounds on the error of a
32-bit evaluation.

u = 2^-24 is the unit of an fp32 rounding.  A sum of n fp32 terms, in any order,
is off by at most n u times the sum of the magnitudes.
"""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
F64 = torch.float64


def embed_grad(ids, dout, V, scale):
    """(gradient [V, D], bound of its error per element)."""
    D = dout.shape[1]
    ok = (ids >= 0) & (ids < V)
    i, d = ids[ok].long(), dout[ok].double()
    g = torch.zeros(V, D, dtype=F64).index_add_(0, i, d)
    mag = torch.zeros(V, D, dtype=F64).index_add_(0, i, d.abs())
    n = torch.bincount(i, minlength=V).double()[:, None]
    return g * scale, (n + 2.0) * U * mag * abs(scale)


def logp(z, y, V):
    """(log p(y_t), softmax) of the first V columns; NaN for a target outside them."""
    zd = z[:, :V].double()
    ls = torch.log_softmax(zd, 1)
    ok = (y >= 0) & (y < V)
    lp = ls[torch.arange(z.shape[0]), torch.where(ok, y, 0).long()]
    return torch.where(ok, lp, torch.nan), ls.exp()


def logp_bound(z, y, V):
    """|error| of a 32-bit logp: the difference z_y - m and the log each round; the sum
    of exponentials s is off relatively by its additions (a thread adds V / 256 terms
    at least, then a tree of 10) and its terms (the argument's rounding, at most
    u |x| exp(x) <= 0.4 u of a sum that holds exp(0) for every one, and 2 ulp of exp)."""
    zd = z[:, :V].double()
    m = zd.amax(1)
    zy = zd[torch.arange(z.shape[0]), y.clamp(0, V - 1).long()]
    ls = (zd - m[:, None]).exp().sum(1).log()
    x = (m[:, None] - zd).clamp(max=100.0)
    arg = (x * (-x).exp()).sum(1) / ls.exp()
    return 2 * U * (m - zy).abs() + 4 * U * ls + (V / 256 + 10 + 8 + 4 * arg) * U


def policy(z, y, V, w, adv, old, ref, lo, hi, kl):
    """(loss, logp, c, softmax): c is dloss/dlogp."""
    lp, p = logp(z, y, V)
    live = w != 0
    lp = torch.where(live, lp, 0.0)
    ratio = (lp - old.double()).exp()
    A = adv.double()
    free, held = ratio * A, ratio.clamp(1.0 - lo, 1.0 + hi) * A
    loss = -torch.where(held < free, held, free)
    g = torch.where(held < free, 0.0, -free)
    if kl:
        d = ref.double() - lp
        loss = loss + kl * (torch.expm1(d) - d)
        g = g - kl * torch.expm1(d)
    wd = w.double()
    return torch.where(live, wd * loss, 0.0).sum(), lp, torch.where(live, wd * g, 0.0), p


def preference(z, y, V, w, ref, seq, beta, eps):
    """(loss, margins, logp, c, softmax)."""
    lp, p = logp(z, y, V)
    live = w != 0
    lp = torch.where(live, lp, 0.0)
    x = torch.where(live, w.double() * (lp - (0.0 if ref is None else ref.double())), 0.0)
    P = (len(seq) - 1) // 2
    c, margins, total = torch.zeros_like(lp), [], 0.0
    for i in range(P):
        a, b, d = seq[2 * i:2 * i + 3]
        m = beta * float(x[a:b].sum() - x[b:d].sum())
        margins.append(m)
        total += (1.0 - eps) * math.log1p(math.exp(-m)) + eps * math.log1p(math.exp(m))
        g = beta / P * (1.0 / (1.0 + math.exp(-m)) - (1.0 - eps))
        c[a:b], c[b:d] = g, -g
    c = torch.where(live, w.double() * c, 0.0)
    return total / P, torch.tensor(margins, dtype=F64), lp, c, p


def dlogits(c, p, y, ld):
    """c_t ([j = y_t] - p_tj), zeros in the padding columns and where c is 0."""
    T, V = p.shape
    d = torch.zeros(T, ld, dtype=F64)
    on = c != 0
    d[:, :V] = torch.where(on[:, None], -c[:, None] * p, 0.0)
    ok = (y >= 0) & (y < V) & on
    d[torch.nonzero(ok)[:, 0], y[ok].long()] += c[ok]
    return d


def clip(grads, max_norm):
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    c = 1.0 if norm <= max_norm else max_norm / norm
    return norm, c, [g.double() * c for g in grads]
