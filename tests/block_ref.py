"""float64 references (CPU) for the operators of include/qblock.h, written from their definitions, with
elementwise error bounds.

Bounds.  U32 = 2^-24, and a type's unit, are half a step relative to the value (head_ref.py).  A sum whose
values pass through at most d additions each is off by at most d U32 sum |v| to first order, products by n for
n terms in any order.  DEPTH is the longest chain in the norm's kernels: 128 values of a thread (or 64 and 16 batches of them), the lanes
of a wave (6), eight waves, the entries of a group a lane takes (up to 64), the partial sums' joining.
"""
from __future__ import annotations

import math

import torch

from head_ref import U32, act, near, slope, unit  # noqa: F401

DEPTH = 320
KEEP = 32


def pack(x):
    """(q, e, x8) of a matrix, from the definition, in integers and float64."""
    rows, cols = x.shape
    q = torch.zeros(rows, cols, dtype=torch.int8)
    e = torch.zeros(rows, -(-cols // KEEP), dtype=torch.uint8)
    x8 = torch.zeros(rows, cols, dtype=torch.float64)
    for b in range(e.shape[1]):
        v = x[:, b * KEEP:(b + 1) * KEEP].double()
        for r in range(rows):
            row = v[r]
            at = (r, slice(b * KEEP, b * KEEP + row.numel()))
            if not bool(torch.isfinite(row).all()):
                e[r, b] = 255
                x8[at] = math.nan
                continue
            top, E = row.abs().max().item(), -126
            if top > 0:
                E = max(-126, math.frexp(top)[1] - 8)
                while 127 * 2.0 ** E < top:
                    E += 1
            n = torch.round(row / 2.0 ** E)  # (exact quotients; torch rounds halves to even)
            if E == 122:
                n = n.clamp(-63, 63)
            e[r, b] = E + 127
            q[at] = n.to(torch.int8)
            x8[at] = n * 2.0 ** E
    return q, e, x8


def unpack(q, e):
    scale = torch.exp2(e.double() - 127).masked_fill(e == 0, 0.0).masked_fill(e == 255, math.nan)
    return q.double() * scale.repeat_interleave(KEEP, dim=-1)[..., : q.shape[-1]]


# --- group norm: x (n, p, c) -----------------------------------------------------------

def _split(t, groups):
    n, p, c = t.shape
    return t.double().view(n, p, groups, c // groups)


def _wide(t, like):
    return t.double().view(1, 1, *like.shape[2:]) if t is not None else None


def _avg(t):
    return t.mean(dim=(1, 3), keepdim=True)


def norm(x, groups, gamma, beta, eps, name):
    """{y, mean, rstd: (value, bound before rounding)}."""
    v = _split(x, groups)
    mean = _avg(v)
    d = v - mean
    var = _avg(d * d)
    rstd = 1 / torch.sqrt(var + eps)
    em = DEPTH * U32 * _avg(v.abs()) + 2 * U32 * mean.abs()
    # (x - m')^2 averages to var + (m - m')^2; each difference is rounded once, beside values up to |x - mean| + em
    rel = ((DEPTH + 8) * U32 * var + em * em) / (var + eps)
    er = rstd * (0.5 * rel + 4 * U32)
    xh = d * rstd
    ga, be = (_wide(gamma, v) if gamma is not None else 1.0), (_wide(beta, v) if beta is not None else 0.0)
    z = xh * ga + be
    ex = em * rstd + xh.abs() * (er / rstd + 4 * U32)
    g = torch.as_tensor(ga).abs()
    ez = g * ex + 3 * U32 * (z.abs() + (xh * g).abs())
    y = act(z, name)
    ey = 1.13 * ez + (0 if name == "none" else 16 * U32 * (1 + z.abs()))
    n = x.shape[0]
    return {"y": (y.reshape(x.shape), ey.reshape(x.shape)), "mean": (mean.view(n, groups), em.view(n, groups)),
            "rstd": (rstd.view(n, groups), er.view(n, groups))}


def norm_grads(dy, x, groups, gamma, beta, mean, rstd, name):
    """{dx, dgamma, dbeta: (value, bound)} for given statistics (float32); x may be what a checkpoint stands for."""
    v, dy4, n = _split(x, groups), _split(dy, groups), x.shape[0]
    c = x.shape[2]
    m, r = mean.double().view(n, 1, groups, 1), rstd.double().view(n, 1, groups, 1)
    ga = _wide(gamma, v) if gamma is not None else torch.ones(())
    be = _wide(beta, v) if beta is not None else torch.zeros(())
    xh = (v - m) * r
    ex = 3 * U32 * xh.abs()
    z = xh * ga + be
    ez = ga.abs() * ex + 3 * U32 * (z.abs() + (xh * ga).abs())
    s = slope(z, name) if name != "none" else torch.ones_like(z)
    dz = dy4 * s
    # |act''| <= 1.2; the slope itself costs a dozen roundings of terms up to 1 + |z|
    edz = torch.zeros_like(dz) if name == "none" else dy4.abs() * (1.2 * ez + 32 * U32 * (1 + z.abs()))
    t, et = ga * dz, ga.abs() * edz + U32 * (ga * dz).abs()
    a, b = _avg(t), _avg(t * xh)
    ea = _avg(et) + DEPTH * U32 * _avg(t.abs())
    eb = _avg(et * xh.abs() + t.abs() * ex) + DEPTH * U32 * _avg((t * xh).abs())
    dx = r * (t - a - xh * b)
    edx = r * (et + ea + xh.abs() * eb + ex * b.abs() + 6 * U32 * (t.abs() + a.abs() + (xh * b).abs()))

    def sums(w, ew):
        return w.sum(dim=(0, 1)).view(c), (ew.sum(dim=(0, 1)) + DEPTH * U32 * w.abs().sum(dim=(0, 1))).view(c)

    return {"dx": (dx.reshape(x.shape), edx.reshape(x.shape)), "dgamma": sums(dz * xh, edz * xh.abs() + dz.abs() * ex),
            "dbeta": sums(dz, edz)}


# --- gated layer -----------------------------------------------------------------------

def gated(x, wg, wu, bg, bu, name):
    """{h, g, u: (value, bound)}."""
    def one(w, b):
        z = x.double() @ w.double().t() + (b.double() if b is not None else 0.0)
        mass = x.double().abs() @ w.double().abs().t() + (b.double().abs() if b is not None else 0.0)
        return z, (x.shape[1] + 8) * U32 * mass

    (g, eg), (u, eu) = one(wg, bg), one(wu, bu)
    a = act(g, name)
    ea = 1.13 * eg + (0 if name == "none" else 16 * U32 * (1 + g.abs()))
    return {"h": (a * u, ea * u.abs() + a.abs() * eu + ea * eu + U32 * (a * u).abs()), "g": (g, eg), "u": (u, eu)}


def gated_grads(x, wg, wu, dh, g, u, name, dtype):
    """{dx, dwg, dwu, dbg, dbu: (value, bound)} from g and u as the backward has them; dg and du are rounded to dtype."""
    ut = unit(dtype)
    x, wg, wu, dh, g, u = (t.double() for t in (x, wg, wu, dh, g, u))
    s = slope(g, name) if name != "none" else torch.ones_like(g)
    dg, du = dh * u * s, dh * act(g, name)
    zero = name == "none"
    edg = 2 * U32 * dg.abs() + (0 if zero else 32 * U32 * (dh * u).abs() * (1 + g.abs()))
    edu = U32 * du.abs() + (0 if zero else 16 * U32 * dh.abs() * (1 + g.abs()))
    m, n = dh.shape
    pg, pu = edg + ut * (dg.abs() + edg), edu + ut * (du.abs() + edu)
    out = {"dx": (dg @ wg + du @ wu, pg @ wg.abs() + pu @ wu.abs() + (2 * n + 8) * U32 * (dg.abs() @ wg.abs() + du.abs() @ wu.abs()))}
    for k, d, e, p in (("g", dg, edg, pg), ("u", du, edu, pu)):
        out["dw" + k] = d.t() @ x, p.t() @ x.abs() + (m + 8) * U32 * (d.abs().t() @ x.abs())
        out["db" + k] = d.sum(0), e.sum(0) + (m + 8) * U32 * d.abs().sum(0)
    return out
