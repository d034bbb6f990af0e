"""What stands between the linears from its definitions, in 64 bits on the CPU (plain
torch; shares nothing with the package), and bounds on the error of a 32-bit
evaluation.

u = 2^-24 is the unit of an fp32 rounding; an output of type t is off by half a step more,
torch.finfo(t).eps / 2 of its size.
"""
from __future__ import annotations

import torch

U = 2.0 ** -24
F64 = torch.float64
GROUP = 128


# ---- activations in 8 bits -----------------------------------------------------------
def act8(x):
    """(codes, scale) of x by the definition; codes from quotients in 64 bits, which lie at
    least 2^-33 from a half that they are not on (24-bit operands), scale in fp32."""
    T, D = x.shape
    n = -(-D // GROUP)
    codes, scale = torch.zeros(T, D, dtype=torch.int8), torch.zeros(T, n)
    for k in range(n):
        part = x[:, k * GROUP:(k + 1) * GROUP].double()
        finite = part.isfinite().all(1)
        part = torch.where(finite[:, None], part, 0.0)
        m = part.abs().amax(1)
        q = torch.floor(part.abs() * 127.0 / torch.where(m > 0, m, 1.0)[:, None] + 0.5) * part.sign()
        codes[:, k * GROUP:(k + 1) * GROUP] = q.to(torch.int8)
        scale[:, k] = torch.where(finite, m.float() / 127.0, torch.nan)
    return codes, scale


def act8_values(codes, scale):
    return codes.double() * scale.double().repeat_interleave(GROUP, 1)[:, : codes.shape[1]]


# ---- the LoRA backward from them -------------------------------------------------------
def linear_bwd(xq, W, A, B, u, dy, s):
    """(dx, dA, dB) in 64 bits, u None: recomputed."""
    dy, A, B = dy.double(), A.double(), B.double()
    u = xq @ A.T if u is None else u.double()
    du = s * (dy @ B)
    return dy @ W.double() + du @ A, du.T @ xq, s * (dy.T @ u)


def linear_bwd_bounds(xq, W, A, B, u, dy, s):
    """Bounds of the error of (dx, dA, dB).  du and u: sums of N (K) fp32 terms, which are exact
    products.  dx: their sum and du's rounding to bf16, then its own.  dA: du times
    x's scale, rounded, as three bf16 (each half a step, 2^-9, of what the one before left: 2^-27 at the end),
    times whole numbers, three sums over T in one."""
    T, K = xq.shape
    N = dy.shape[1]
    dyd, Ad, Bd = dy.double().abs(), A.double().abs(), B.double().abs()
    mag_u = xq.abs() @ Ad.T if u is None else u.double().abs()
    du_err = abs(s) * (N + 3) * U * (dyd @ Bd)
    u_err = (K + 3) * U * mag_u if u is None else torch.zeros_like(mag_u)
    mag_du = abs(s) * (dyd @ Bd)
    split = 2.0 ** -27 + U
    dx_mag = dyd @ W.double().abs() + mag_du @ Ad
    dx = (N + 8 + A.shape[0]) * U * dx_mag + (du_err + 2.0 ** -8 * mag_du) @ Ad
    dA = (du_err + (split + (3 * T + 8) * U) * mag_du).T @ xq.abs()
    dB = abs(s) * (dyd.T @ (u_err + (split + (3 * T + 8) * U) * mag_u))
    return dx, dA, dB


# ---- norms, gate and residual sum ------------------------------------------------------
# Roundings on the way to the reciprocal root of a row's mean square: up to 16 squares a thread,
# 6 levels of a wave, 16 waves, then mean, eps, root and reciprocal, the root halving what
# came before.
ROOT = 23.0
# ... and of a sum over a row of products: 16 + 6 + 16, the product and the mean.
SUM = 42.0


def _gain(w, off, D):
    return torch.ones(D, dtype=F64) if w is None else w.double() + off


def norm_fwd(h, y, post, w_post, gate, w_pre, eps, off, a):
    """dict of h, n, rstd_post, rstd_pre (64 bits), and of their bounds before the outputs' rounding."""
    D = h.shape[1]
    h = h.double()
    out, err = {}, {}
    if y is not None:
        yn, rel = y.double(), 0.0
        if post:
            r2 = 1.0 / torch.sqrt(yn.square().mean(1, keepdim=True) + eps)
            out["rstd_post"], err["rstd_post"] = r2[:, 0], ROOT * U * r2[:, 0]
            yn, rel = yn * r2 * _gain(w_post, off, D), ROOT + 3.0
        part = a * yn * (1.0 if gate is None else gate.double())
        hn = h + part
        eh = (rel + 2.0) * U * part.abs() + U * hn.abs()
    else:
        hn, eh = h, torch.zeros_like(h)
    r1 = 1.0 / torch.sqrt(hn.square().mean(1, keepdim=True) + eps)
    # the root's own roundings, and what the stream's errors move it
    moved = (hn.abs() * eh).mean(1, keepdim=True) * r1 ** 2
    n = hn * r1 * _gain(w_pre, off, D)
    out["h"], err["h"] = hn, eh
    out["rstd_pre"], err["rstd_pre"] = r1[:, 0], ((ROOT * U + moved) * r1)[:, 0]
    out["n"] = n
    err["n"] = (ROOT * U + moved + 3.0 * U) * n.abs() + eh * r1 * _gain(w_pre, off, D).abs()
    return out, err


def norm_bwd(dn, dh_out, h, y, post, w_post, gate, w_pre, r2, r1, off, a):
    """dict of dh, dy, dw_pre, dw_post, dgate, and of their bounds before the outputs' rounding.
    h and y as values in 64 bits; r1, r2 [T] as given.  A sum over a row of weights k times dh may be
    taken in two parts, dh = p - q hh with q = r1 c: sum k p - q sum k hh, whose terms are up to
    |k dh| + 2 |k q hh| together."""
    like = dn if dn is not None else dh_out
    T, D = like.shape
    over_rows = (T / 32.0 + 64.0) * U  # a sum over rows: rows of a workgroup in turn, then 512 sums in 16 ranges
    out, err = {}, {}
    dh = torch.zeros(T, D, dtype=F64) if dh_out is None else dh_out.double()
    eh = torch.zeros(T, D, dtype=F64)
    parts = torch.zeros(T, D, dtype=F64)  # 2 |q hh|
    if dn is not None:
        hh, e = h.double() * r1.double()[:, None], dn.double() * _gain(w_pre, off, D)
        c = (e * hh).mean(1, keepdim=True)
        ec = (SUM + 3.0) * U * (e * hh).abs().mean(1, keepdim=True)
        r = r1.double()[:, None].abs()
        eh = r * (4.0 * U * e.abs() + hh.abs() * ec + 4.0 * U * (hh * c).abs())
        dh = dh + r1.double()[:, None] * (e - hh * c)
        eh = eh + U * dh.abs()
        parts = 2.0 * r * (hh * c).abs()
        out["dw_pre"] = (dn.double() * hh).sum(0)
        err["dw_pre"] = (over_rows + 3.0 * U) * (dn.double() * hh).abs().sum(0)
    out["dh"], err["dh"] = dh, eh
    g = torch.ones(1, 1, dtype=F64) if gate is None else gate.double()
    w2 = _gain(w_post, off, D) if post else torch.ones(D, dtype=F64)
    z, ez = a * dh, abs(a) * eh + U * (a * dh).abs()
    if y is not None:
        yh = y.double() * r2.double()[:, None] if post else y.double()
        per = z * yh * w2
        eper = ez * (yh * w2).abs() + 4.0 * U * per.abs()
        if gate is not None:
            if gate.shape == (D,):
                out["dgate"], err["dgate"] = per.sum(0), (eper + over_rows * per.abs()).sum(0)
            elif gate.shape == (T, 1):
                out["dgate"] = per.sum(1, keepdim=True)
                err["dgate"] = (eper + (SUM + 3.0) * U * (per.abs() + abs(a) * parts * (yh * w2).abs())).sum(1, keepdim=True)
            else:
                out["dgate"], err["dgate"] = per, eper
        if post:
            out["dw_post"] = (z * g * yh).sum(0)
            err["dw_post"] = ((ez * g.abs() * yh.abs()) + (3.0 * U + over_rows) * (z * g * yh).abs()).sum(0)
    f, ef = z * g * w2, (ez * (g * w2).abs() + 3.0 * U * (z * g * w2).abs())
    if post:
        c = (f * yh).mean(1, keepdim=True)
        ec = (ef * yh.abs() + (SUM + 3.0) * U * ((f * yh).abs() + abs(a) * parts * (g * w2 * yh).abs())).mean(1, keepdim=True)
        r = r2.double()[:, None]
        out["dy"] = r * (f - yh * c)
        err["dy"] = r.abs() * (ef + yh.abs() * ec + 4.0 * U * (f.abs() + (yh * c).abs()))
    else:
        out["dy"], err["dy"] = f, ef
    return out, err


def check(got, want, err, name=""):
    """Every element within its bound and the rounding to its own type; not finite where, and as, the
    definition is not."""
    g = got.detach().cpu()
    half = torch.finfo(g.dtype).eps / 2
    tiny = torch.finfo(g.dtype).tiny  # (below it a step is not relative)
    w = want.reshape(g.shape)
    bound = err.reshape(g.shape) * (1.0 + half) + half * w.abs() + tiny
    g = g.double()
    fine = w.isfinite()
    assert torch.equal(g.isfinite(), fine), f"{name}: {int((g.isfinite() != fine).sum())} values finite or not where they should not be"
    off = torch.where(fine, (g - w).abs() - bound, 0.0)
    assert float(off.max()) <= 0.0, f"{name}: {float(off.max()):.3g} past the bound, {int((off > 0).sum())} of {off.numel()}"
