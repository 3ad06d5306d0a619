"""Plain 64-bit forms of the feed-forward and gradient operators, and the
largest error that the library's roundings allow, derived value by value.

Notation: u is the unit roundoff of the tensors' type (2^-8 for bfloat16,
2^-11 for float16), e = 2^-24 that of fp32. A product over k terms summed in
fp32 in any order is off by at most k e sum|a b|; an activation computed in
fp32 by at most 64 e (|z| + 1) (a few roundings, exp and erf of 2 ulp, whose
argument's own rounding the factor |z| covers); an output rounded once by
u |y|, or half the smallest subnormal.
"""
from __future__ import annotations

import math

import torch

E = 2.0 ** -24


def unit(dtype):
    return 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11


def tiny(dtype):
    return 2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134


def act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z * math.sqrt(0.5))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))


def act_grad(name, z):
    if name == "none":
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * torch.special.erfc(-z * math.sqrt(0.5)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)


def act_error(z):
    """of an activation and of its derivative, from fp32 arithmetic"""
    return 64 * E * (z.abs() + 1)


SLOPE = 1.13   # the largest derivative of the activations


def rounded(y, err, dtype):
    """the bound of an output: its own rounding on top of what it is rounded from"""
    return err + unit(dtype) * (y.abs() + err) + tiny(dtype)


def linear(x, w, bias, name, residual, dtype):
    """(y, bound of y, z, bound of z), z before the activation"""
    x, w = x.double(), w.double()
    k = x.shape[1]
    z = x @ w.t()
    ez = (k + 4) * E * (x.abs() @ w.abs().t())
    if bias is not None:
        z = z + bias.double()
        ez = ez + 4 * E * z.abs()
    y = act(name, z)
    ey = SLOPE * ez + (act_error(z) if name != "none" else 0)
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2 * E * y.abs()
    return y, rounded(y, ey, dtype), z, rounded(z, ez, dtype)


def linear_backward(dy, x, w, name, z, dtype):
    """{name: (gradient, bound)} from the z that was kept"""
    dy, x, w = dy.double(), x.double(), w.double()
    if name == "none":
        dz, ed = dy, torch.zeros_like(dy)
    else:
        dz = dy * act_grad(name, z.double())
        ed = rounded(dz, dy.abs() * act_error(z.double()) + 2 * E * dz.abs(), dtype)   # dz is rounded as an operand
    m, n = dz.shape
    one = torch.ones(1, m, dtype=torch.float64, device=dz.device)
    out = {}
    for key, a, ea, b in (("dx", dz, ed, w), ("dw", dz.t(), ed.t(), x)):
        c = a @ b
        out[key] = (c, rounded(c, (a.shape[1] + 4) * E * (a.abs() @ b.abs()) + 1.01 * (ea @ b.abs()), dtype))
    c = (one @ dz)[0]
    out["db"] = (c, rounded(c, ((m + 4) * E * (one @ dz.abs()) + 1.01 * (one @ ed))[0], dtype))
    return out


def ffn(x, w_in, w_out, name, residual, dtype):
    """(y, bound, p, bound of p)"""
    x, w_in, w_out = x.double(), w_in.double(), w_out.double()
    f, d = w_out.shape[1], x.shape[1]
    p = x @ w_in.t()
    ep = (d + 4) * E * (x.abs() @ w_in.abs().t())
    g, u = p[:, :f], p[:, f:]
    h = act(name, g) * u
    eh = (SLOPE * ep[:, :f] + act_error(g)) * (u.abs() + ep[:, f:]) + act(name, g).abs() * ep[:, f:] + 2 * E * h.abs()
    eh = rounded(h, eh, dtype)
    y = h @ w_out.t()
    ey = (f + 4) * E * (h.abs() @ w_out.abs().t()) + 1.01 * (eh @ w_out.abs().t())
    if residual is not None:
        y = y + residual.double()
        ey = ey + 2 * E * y.abs()
    return y, rounded(y, ey, dtype), p, rounded(p, ep, dtype)


def ffn_backward(dy, x, w_in, w_out, name, p, dtype):
    """{name: (gradient, bound)} from the p that was kept"""
    dy, x, w_in, w_out, p = dy.double(), x.double(), w_in.double(), w_out.double(), p.double()
    f = w_out.shape[1]
    d, t = x.shape[1], x.shape[0]
    g, u = p[:, :f], p[:, f:]
    a, da = act(name, g), act_grad(name, g)
    h = a * u
    eh = rounded(h, act_error(g) * u.abs() + 2 * E * h.abs(), dtype)
    dh = dy @ w_out
    edh = (d + 4) * E * (dy.abs() @ w_out.abs())
    dg, du = dh * u * da, dh * a
    edg = edh * (u * da).abs() + (dh.abs() + edh) * u.abs() * act_error(g) + 4 * E * dg.abs()
    edu = edh * a.abs() + (dh.abs() + edh) * act_error(g) + 4 * E * du.abs()
    dp = torch.cat([dg, du], 1)
    edp = rounded(dp, torch.cat([edg, edu], 1), dtype)
    out = {}
    for key, q, eq, b, eb in (("dx", dp, edp, w_in, None), ("dw_in", dp.t(), edp.t(), x, None),
                              ("dw_out", dy.t(), None, h, eh)):
        c = q @ b
        e = (q.shape[1] + 4) * E * (q.abs() @ b.abs())
        if eq is not None:
            e = e + 1.01 * (eq @ b.abs())
        if eb is not None:
            e = e + 1.01 * (q.abs() @ eb)
        out[key] = (c, rounded(c, e, dtype))
    return out


def over_groups(offsets, rows, fn):
    """fn(e, slice of rows) for every expert group, as a list"""
    return [fn(e, slice(offsets[e], offsets[e + 1])) for e in range(len(offsets) - 1)]
