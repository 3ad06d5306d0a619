"""Plain 64-bit forms of attention, layer normalisation and expert balance, and
the largest error that the library's roundings allow, derived value by value.

u, e, tiny and rounded are those of ffn_reference: an output is rounded once by
u relative to the value, fp32 arithmetic by e = 2^-24, a sum of k products in
any order by k e sum|a b|. exp2, log2, the reciprocal and the square root's are
of 1 ulp: 2 e each.
"""
from __future__ import annotations

import math

import torch

from ffn_reference import E, rounded, tiny, unit


# values below 2^-126 may count as zero: exp2 and the matrix cores take subnormal fp32 and bf16 values so
FLUSH = 2.0 ** -126


def visible(lq, lk, causal, prefix, device):
    at = torch.arange(lq, device=device)[:, None] + (lk - lq)
    j = torch.arange(lk, device=device)[None]
    seen = torch.ones(lq, lk, dtype=torch.bool, device=device)
    if causal:
        seen = (j <= at) | (j < prefix)
    return seen, (at - j).abs().double()


def scores(q, k, scale, cap, slope, seen, distance):
    """(scores with -inf where hidden, bound of their error, tanh or None, its error). 16 e: the products'
    sum is scaled, capped and biased by a few roundings of values of at most |z| + |cap| + |bias|;
    the tanh is 1 - 2 / (1 + e^u): absolute errors of the ends' 8 e (a reciprocal, an exponential
    whose argument is off by e |u| and whose slope is at most 1/4, and the difference)."""
    z = q @ k.t() * scale
    ez = (q.shape[1] + 4) * E * (q.abs() @ k.abs().t()) * scale + 4 * E * z.abs()
    t = et = None
    if cap:
        t = torch.tanh(z / cap)
        et = ez / cap + 8 * E
        z, ez = cap * t, cap * et + 4 * E * cap
    if slope is not None:
        z = z - slope * distance
        ez = ez + 8 * E * (slope * distance + z.abs())
    return torch.where(seen, z, torch.full_like(z, -math.inf)), ez, t, et


def attention(q, k, v, dtype, scale, causal=False, cap=0.0, slope=None, prefix=0):
    """One head of one sequence: (y, bound, lse, bound)"""
    q, k, v = q.double(), k.double(), v.double()
    lq, lk = q.shape[0], k.shape[0]
    seen, distance = visible(lq, lk, causal, prefix, q.device)
    if lk == 0 or lq == 0:
        none = q.new_full((lq,), -math.inf)
        return torch.zeros(lq, v.shape[1], dtype=torch.float64, device=q.device), q.new_zeros(lq, v.shape[1]), none, none.new_zeros(lq)
    z, ez, _, _ = scores(q, k, scale, cap, slope, seen, distance)
    lse = torch.logsumexp(z, 1)
    any_ = seen.any(1)
    p = torch.where(any_[:, None], torch.exp(z - torch.where(any_, lse, torch.zeros_like(lse))[:, None]), torch.zeros_like(z))
    # an exponent of 2 is formed from z and a maximum of the size of the row's largest score
    zs = torch.where(seen, z, torch.zeros_like(z))
    large = zs.abs().amax(1, keepdim=True)
    ep = ez + 4 * E * (zs.abs() + large + 1) + 4 * E
    el = (p * ep).sum(1) + (lk + 4) * E                       # of the sum, relative
    y = p @ v
    # p is rounded to the operands' type; it is kept relative to a maximum that is at most 2^8 behind: p >= 1 somewhere
    ey = (p * (ep + unit(dtype))) @ v.abs() + (tiny(dtype) * seen.double()) @ v.abs() + (lk + 4) * E * (p @ v.abs()) + el[:, None] * y.abs()
    elog = torch.where(any_, el + 8 * E * (lse.abs() + large[:, 0] + 1), torch.zeros_like(el))
    return y, torch.where(any_[:, None], rounded(y, 1.01 * ey, dtype), torch.zeros_like(y)), lse, 1.01 * elog


def attention_backward(dy, q, k, v, y, lse, else_, dtype, scale, causal=False, cap=0.0, slope=None, prefix=0):
    """One head of one sequence, from the y that was kept: {name: (gradient, its error before rounding)}. lse: the
    exact one, the kept one is off by else_"""
    dy, q, k, v, y = (t.double() for t in (dy, q, k, v, y))
    lq, lk = q.shape[0], k.shape[0]
    if lk == 0 or lq == 0:
        return {n: (torch.zeros_like(t), torch.zeros_like(t)) for n, t in (("dq", q), ("dk", k), ("dv", v))}
    seen, distance = visible(lq, lk, causal, prefix, q.device)
    z, ez, t, et = scores(q, k, scale, cap, slope, seen, distance)
    any_ = seen.any(1)
    base = torch.where(any_, lse, torch.zeros_like(lse))[:, None]
    p = torch.where(seen, torch.exp(z - base), torch.zeros_like(z))
    zs = torch.where(seen, z, torch.zeros_like(z))
    ep = p * (ez + else_[:, None] + 4 * E * (zs.abs() + base.abs() + 1) + 4 * E) * 1.01 + FLUSH
    dp = dy @ v.t()
    edp = (v.shape[1] + 4) * E * (dy.abs() @ v.abs().t())
    delta = (dy * y).sum(1, keepdim=True)
    edelta = (v.shape[1] + 4) * E * (dy * y).abs().sum(1, keepdim=True)
    ds = p * (dp - delta)
    eds = ep * (dp - delta).abs() + (p + ep) * (edp + edelta + 2 * E * (dp.abs() + delta.abs())) + 4 * E * ds.abs()
    if t is not None:
        f = 1 - t * t
        eds = eds * (f + 2 * t.abs() * et + et * et + 4 * E) + ds.abs() * (2 * t.abs() * et + et * et + 4 * E)
        ds = ds * f
    both = lambda x, ex: torch.where(seen, ex + unit(dtype) * (x.abs() + ex) + tiny(dtype) + FLUSH, torch.zeros_like(x))  # noqa: E731
    eds, epr = both(ds, eds), both(p, ep)

    def product(a, ea, b, n):
        return a @ b, (n + 4) * (E * (a.abs() @ b.abs()) + FLUSH) + 1.01 * (ea @ b.abs())

    dq, edq = product(ds, eds, k, lk)
    dk, edk = product(ds.t(), eds.t(), q, lq)
    dv, edv = product(p.t(), epr.t(), dy, lq)
    return {"dq": (scale * dq, scale * edq + 2 * E * (scale * dq).abs()), "dk": (scale * dk, scale * edk + 2 * E * (scale * dk).abs()),
            "dv": (dv, edv)}


def layer_norm(x, w, bias, eps, dtype, wdtype):
    """(y, bound, stats, bound): the mean is off by (n + 2) e mean|x|, the differences by that and a
    rounding, the variance by twice their relative error and its sum's; the sums' order is unknown."""
    x = x.double()
    n = x.shape[1]
    mean = x.mean(1, keepdim=True)
    em = (n + 2) * E * x.abs().mean(1, keepdim=True)
    d = x - mean
    ed = em + E * d.abs()
    var = (d * d).mean(1, keepdim=True)
    ev = (2 * d.abs() * ed + ed * ed).mean(1, keepdim=True) + (n + 4) * E * var
    rstd = (var + eps) ** -0.5
    er = rstd * (0.5 * ev / (var + eps) * 1.5 + 8 * E)
    xh = d * rstd
    exh = ed * rstd + d.abs() * er + 2 * E * xh.abs()
    wd, bd = (1.0 if w is None else w.double()), (0.0 if bias is None else bias.double())
    y = xh * wd + bd
    ey = exh * (wd if isinstance(wd, float) else wd.abs()) + 4 * E * ((xh * wd).abs() + abs(bd))
    return y, rounded32(y, 1.01 * ey, dtype), torch.cat([mean, rstd], 1), torch.cat([em + 2 * E * mean.abs(), er * 1.01], 1)


def rounded32(y, err, dtype):
    if dtype == torch.float32:
        return err + E * (y.abs() + err) + 2.0 ** -149
    return rounded(y, err, dtype)


def layer_norm_backward(dy, x, w, stats, residual, dtype, wdtype):
    """{name: (gradient, bound)} from the stats that were kept"""
    x, dy = x.double(), dy.double()
    m, n = x.shape
    mean, rstd = stats.double()[:, :1], stats.double()[:, 1:]
    wd = torch.ones(n, dtype=torch.float64, device=x.device) if w is None else w.double()
    xh = (x - mean) * rstd
    exh = 3 * E * xh.abs() + E * (x - mean).abs() * rstd
    g = dy * wd
    a, b = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    ea = (n + 3) * E * g.abs().mean(1, keepdim=True)
    eb = (n + 4) * E * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * exh).mean(1, keepdim=True)
    dx = rstd * (g - a - xh * b)
    edx = rstd * (ea + xh.abs() * eb + exh * b.abs() + 6 * E * (g.abs() + a.abs() + (xh * b).abs()))
    if residual is not None:
        dx = dx + residual.double()
        edx = edx + 2 * E * (dx.abs() + residual.double().abs())
    out = {"dx": (dx, rounded32(dx, 1.01 * edx, dtype))}
    dw, db = (dy * xh).sum(0), dy.sum(0)
    out["dw"] = (dw, rounded32(dw, (m + 4) * E * (dy * xh).abs().sum(0) + (dy.abs() * exh).sum(0), wdtype))
    out["db"] = (db, rounded32(db, (m + 4) * E * dy.abs().sum(0), wdtype))
    return out


def balance(logits, picked, scale):
    """(counts, rows, mean, its bound, loss, its bound): a probability is off by e (|z - top| + 8 + experts) relative to it"""
    z = logits.double()
    t, n = z.shape
    inside = (picked >= 0) & (picked < n)
    counts = torch.bincount(picked[inside].long(), minlength=n)
    some = inside.any(1)
    p, ep = probabilities(z)
    p, ep = p[some], ep[some]
    rows = int(some.sum())
    mean = p.sum(0) / max(rows, 1)
    em = (ep.sum(0) + (rows + 4) * E * p.sum(0)) / max(rows, 1)
    total = max(int(counts.sum()), 1)
    loss = scale * n * (counts * mean).sum() / total
    return counts, rows, mean, em, loss, abs(scale) * n * (counts * em).sum() / total + 4 * E * loss.abs()


def probabilities(z):
    top = z.amax(1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    d = z - top
    p = torch.exp(d)
    total = p.sum(1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones_like(total), total)
    ep = p * E * (4 * torch.where(p > 0, d.abs(), torch.zeros_like(d)) + z.shape[1] + 16) + 2.0 ** -126
    # of the sum: the others' errors, weighted
    return p, ep + p * ep.sum(1, keepdim=True)


def balance_backward(logits, picked, counts, rows, dloss, scale, residual, dtype):
    """(gradient, bound)"""
    z, c = logits.double(), counts.double()
    n = z.shape[1]
    p, ep = probabilities(z)
    dot = (p * c).sum(1, keepdim=True)
    edot = (ep * c).sum(1, keepdim=True) + (n + 4) * E * dot
    total = float(c.sum())
    factor = dloss * scale * n / (total * rows) if total and rows else 0.0
    d = factor * p * (c - dot)
    ed = abs(factor) * (ep * (c - dot).abs() + (p + ep) * (edot + 4 * E * (c + dot))) + 4 * E * d.abs()
    some = ((picked >= 0) & (picked < n)).any(1, keepdim=True)
    d, ed = torch.where(some, d, torch.zeros_like(d)), torch.where(some, ed, torch.zeros_like(ed))
    if residual is not None:
        d = d + residual.double()
        ed = ed + 2 * E * (d.abs() + residual.double().abs())
    return d, rounded32(d, 1.01 * ed, dtype)
