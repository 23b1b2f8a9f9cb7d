"""float64 references (CPU) for the operators at the end of a network, written from their
definitions, with elementwise error bounds.

Bounds.  U32 = 2^-24 and U16 = 2^-8 are the unit roundoffs of float32 and bfloat16.  A sum of n
products accumulated in float32 in any order is off by at most n U32 sum |a_i b_i| to first
order; the factors below add a few roundings for what comes before and after a sum.
"""
from __future__ import annotations

import math

import torch

U32, U16 = 2.0 ** -24, 2.0 ** -8
INF, NAN = math.inf, math.nan


def unit(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def act(z, name):
    return {"none": lambda u: u, "relu": torch.relu, "gelu": torch.nn.functional.gelu, "silu": torch.nn.functional.silu,
            "gelu_tanh": lambda u: torch.nn.functional.gelu(u, approximate="tanh")}[name](z)


def slope(z, name):
    z = z.detach().clone().requires_grad_(True)
    return torch.autograd.grad(act(z, name).sum(), z)[0]


def linear(x, w, b, r, name):
    """(y, z, bound of y, bound of z) before the outputs' own rounding."""
    x, w = x.double(), w.double()
    z = x @ w.t() + (b.double() if b is not None else 0.0)
    mass = x.abs() @ w.abs().t() + (b.double().abs() if b is not None else 0.0)
    ez = (x.shape[1] + 8) * U32 * mass
    y = act(z, name)
    # |act'| <= 1.13; evaluating act itself costs a dozen roundings of values up to 1 + |z|
    ey = 1.13 * ez + (0 if name == "none" else 16 * U32 * (1 + z.abs()))
    if r is not None:
        y = y + r.double()
        ey = ey + U32 * y.abs()
    return y, z, ey, ez


def linear_grads(x, w, dy, z, name):
    """{name: (value, bound before the output's rounding)} of dx, dw, db; dz is rounded to the inputs' type."""
    u = unit(x.dtype)
    x, w, dy, z = x.double(), w.double(), dy.double(), z.double()
    dz = dy * slope(z, name) if name != "none" else dy
    # the slope: a dozen roundings of terms up to 1.13 + |z| e^(-z^2/2) ...; then dz to the type of the products
    e = 0 * dz if name == "none" else 32 * U32 * dy.abs() * (1 + z.abs())
    ep = e if name == "none" else e + u * dz.abs()
    n, m = w.shape[0], x.shape[0]
    out = {"dx": (dz @ w, ep @ w.abs() + (n + 8) * U32 * (dz.abs() @ w.abs())),
           "dw": (dz.t() @ x, ep.t() @ x.abs() + (m + 8) * U32 * (dz.abs().t() @ x.abs())),
           "db": (dz.sum(0), e.sum(0) + (m + 8) * U32 * dz.abs().sum(0))}
    return out


def near(got, ref, bound, dtype):
    """got (of dtype) within bound of ref, and its own rounding; where ref is not finite in dtype, equal to it."""
    got, ref = got.detach().double().cpu(), ref.double()
    ref = torch.where(torch.isinf(ref.to(dtype)), ref.to(dtype).double(), ref)
    fine = torch.isfinite(ref)
    # at the very end of the type's range the bound reaches infinity
    at_end = fine & torch.isinf(got) & (ref.sign() == got.sign()) & (ref.abs() * (1 + unit(dtype)) + bound > torch.finfo(dtype).max)
    got = torch.where(at_end, ref, got)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), "NaN in other places"
    assert torch.equal(got[~fine].nan_to_num(7.0), ref[~fine].nan_to_num(7.0)), "infinities in other places"
    over = (got - ref).abs()[fine] - (bound + unit(dtype) * (ref.abs() + bound) + 1e-37)[fine]
    assert over.numel() == 0 or over.max().item() <= 0, f"off by {over.max().item():.3g} more than the bound"


# --- rows of logits ------------------------------------------------------------------

def softmax_parts(z, t):
    """log p, p and lse of z / t by rows; an all -inf row has log p = -inf, p = 0, lse = -inf."""
    u = z.double() / t
    m = u.amax(1, keepdim=True)
    m = torch.where(torch.isinf(m) & (m < 0), torch.zeros_like(m), m)
    ls = torch.log(torch.exp(u - m).sum(1, keepdim=True))
    lse = m + ls
    # (u - m first: beside an m of 1e38 the logarithm would vanish)
    logp = torch.where(torch.isinf(lse) & (lse < 0), torch.full_like(u, -INF), u - m - ls)
    return logp, torch.exp(logp), lse[:, 0]


def rank(z):
    """Indices of each row by falling value, equal ones by rising index, NaN last."""
    key = torch.where(torch.isnan(z), torch.full_like(z, -INF, dtype=torch.float64), z.double())
    nan = torch.isnan(z).long()
    order = torch.sort(key, dim=1, descending=True, stable=True)[1]
    return order.gather(1, torch.sort(nan.gather(1, order), dim=1, stable=True)[1])


def row_eps(vocab):
    """Relative error of a row's sums: at most vocab / 64 + 40 additions in a chain, and the exponentials', whose
    arguments are off by 3 U32 |d| with 2^-|d| |d| < 1 as their weight."""
    return (vocab / 64 + 48) * U32


def logprobs(z, target, t):
    """(logp, entropy, lse, their bounds)."""
    logp, p, lse = softmax_parts(z, t)
    vocab = z.shape[1]
    eps = row_eps(vocab)
    some = target.clamp(0, vocab - 1)[:, None]
    picked = logp.gather(1, some)[:, 0]
    picked = torch.where(target < 0, torch.zeros_like(picked), torch.where(target >= vocab, torch.full_like(picked, NAN), picked))
    # a NaN or +inf spoils its row; a row without a target stays 0 all the same
    spoilt = torch.isnan(z).any(1) | (z == INF).any(1)
    picked = torch.where(spoilt & (target >= 0), torch.full_like(picked, NAN), picked)
    ent = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    ent = torch.where(spoilt, torch.full_like(ent, NAN), ent)
    lse = torch.where(spoilt, torch.full_like(lse, NAN), lse)
    # differences of values up to |z| / t, each rounded a few times
    size = z.double().nan_to_num(0.0, 0.0, 0.0).abs().amax(1) / t
    e1 = eps + 8 * U32 * (lse.nan_to_num(0, 0, 0).abs() + picked.nan_to_num(0, 0, 0).abs() + torch.log(torch.tensor(float(vocab) + 1)))
    mass = torch.where(p > 0, p * logp.abs(), torch.zeros_like(p)).sum(1)
    return picked, ent, lse, e1, eps * (2 + 3 * mass) + 8 * U32 * math.log(vocab + 2), eps + 8 * U32 * size + 8 * U32 * math.log(vocab + 2)


def logprobs_grad(z, target, t, g, h):
    """(dlogits, bound)."""
    logp, p, _ = softmax_parts(z, t)
    vocab = z.shape[1]
    given = (target >= 0) & (target < vocab)
    up = torch.where(given, g.double(), torch.zeros_like(g.double()))[:, None]
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    ent = -plogp.sum(1, keepdim=True)
    hh = h.double()[:, None] if h is not None else torch.zeros_like(up)
    dz = -up * p - hh * (plogp + p * ent)
    one = torch.zeros_like(p).scatter_(1, target.clamp(0, vocab - 1)[:, None], 1.0)
    dz = (dz + up * one) / t
    spoilt = (torch.isnan(z).any(1) | (z == INF).any(1))[:, None] & ((up != 0) | (hh != 0))
    empty = (z == -INF).all(1, keepdim=True)
    dz = torch.where(spoilt, torch.full_like(dz, NAN), torch.where(empty | ((up == 0) & (hh == 0)), torch.zeros_like(dz), dz))
    eps = row_eps(vocab)
    # a probability: the sum's error, and its own exponent's
    ep = p * (2 * eps + 4 * U32 * logp.abs().nan_to_num(0, 0, 0))
    bound = (up.abs() * (ep + 4 * U32 * one) + hh.abs() * (ep * (logp.abs().nan_to_num(0, 0, 0) + ent.abs() + 1) + p * (4 * eps * (1 + ent.abs())))) / t
    return dz, bound.nan_to_num(0, 0, 0) + 4 * U32 * dz.abs().nan_to_num(0, 0, 0)


def in_range(logp):
    """A log probability below float32's range is -inf."""
    return torch.where(logp < torch.finfo(torch.float32).min, torch.full_like(logp, -INF), logp)


def distill(z, ids, tz, label, t, alpha, g):
    """(loss, dlogits, bounds of both)."""
    rows, vocab = z.shape
    zero = torch.zeros(rows, 1, dtype=torch.float64)
    eps = row_eps(vocab)
    loss, dz = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, vocab, dtype=torch.float64)
    eloss, edz = torch.zeros(rows, dtype=torch.float64), torch.zeros_like(dz)
    wrong = torch.zeros(rows, dtype=torch.bool)
    terms = torch.zeros(rows, dtype=torch.bool)

    def err(logp, p):
        return p * (2 * eps + 4 * U32 * logp.abs().nan_to_num(0, 0, 0))

    if ids is not None and ids.shape[1] and alpha > 0:
        there = ids >= 0
        u = torch.where(there, tz.double() / t, torch.full(ids.shape, -INF, dtype=torch.float64))
        logq, q, _ = softmax_parts(u, 1.0)
        ok = there & (ids < vocab)
        wrong |= (there & ~ok).any(1)
        logp, p, lse = softmax_parts(z, t)
        at = ids.clamp(0, vocab - 1)
        lp = in_range(logp.gather(1, at))
        use = ok & (q > 0)
        diff = torch.where(use, logq - lp, torch.zeros_like(q))
        kl = torch.where(use, q * diff, torch.zeros_like(q))
        loss = loss + alpha * t * t * kl.sum(1)
        size = lp.abs().nan_to_num(0, 0, 0) + logq.abs().nan_to_num(0, 0, 0) + lse.abs().nan_to_num(0, 0, 0)[:, None]
        eloss += alpha * t * t * (q * (eps + 200 * U32 * (1 + diff.abs().nan_to_num(0, 0, 0)) + 16 * U32 * size)).sum(1)
        has = (q > 0).any(1, keepdim=True).double()
        spread = torch.zeros_like(p).scatter_add_(1, at, torch.where(ok, q, torch.zeros_like(q)))
        dz = dz + alpha * t * (has * p - spread)
        edz = edz + alpha * t * (has * err(logp, p) + 200 * U32 * spread)
        terms |= has[:, 0] > 0
    if label is not None and alpha < 1:
        given = (label >= 0) & (label < vocab)
        wrong |= label >= vocab
        logp, p, lse = softmax_parts(z, 1.0)
        at = label.clamp(0, vocab - 1)[:, None]
        ce = -in_range(logp.gather(1, at)[:, 0])
        loss = loss + torch.where(given, (1 - alpha) * ce, torch.zeros_like(ce))
        eloss += torch.where(given, (1 - alpha) * (eps + 16 * U32 * (ce.abs() + lse.abs() + 1)), torch.zeros_like(ce)).nan_to_num(0, 0, 0)
        one = torch.zeros_like(p).scatter_(1, at, 1.0)
        gv = given[:, None].double()
        dz = dz + (1 - alpha) * gv * (p - one)
        edz = edz + (1 - alpha) * gv * (err(logp, p) + 4 * U32 * one)
        terms |= given
    spoilt = (torch.isnan(z).any(1) | (z == INF).any(1)) & terms
    loss = torch.where(spoilt | wrong, torch.full_like(loss, NAN), loss)
    up = g.double()[:, None]
    dead = (up == 0) | ~terms[:, None]
    grad = torch.where(dead, torch.zeros_like(dz), torch.where(spoilt[:, None], torch.full_like(dz, NAN), dz * up))
    edz = (edz.nan_to_num(0, 0, 0) + 4 * U32 * dz.abs().nan_to_num(0, 0, 0)) * up.abs()
    del zero
    return loss, grad, eloss.nan_to_num(0, 0, 0), edz
