"""Attention inside packed documents from its formulas in float64, with a bound for each result of a kernel that rounds as described.

A kernel of storage type t may round the probabilities and their gradients to t before the products that consume them, keeps every sum in float32, and rounds its
results to t once.  With u = half a step of t (2^-8 for bfloat16, 2^-24 for float32) and w = 2^-24:
  a score of d products is off by at most (d + 8) w sum |q k| / sqrt(d) (+ the cap's own arithmetic, 16 w cap), the exponent by that and 4 w (|score| + |lse|) more;
  a probability by its exponent's error, relatively, and u;  a sum over n terms adds n w of the terms' magnitudes.
"""
import math

import torch

W = 2.0 ** -24


def tables(T, lengths, prefixes=None, first=0):
    """Visible interval [lo, hi) of every row (empty for rows of no document)."""
    lo, hi = torch.arange(T), torch.arange(T)
    a = first
    for i, n in enumerate(lengths):
        p = min(n, prefixes[i]) if prefixes else 0
        r = torch.arange(a, a + n)
        lo[a:a + n] = a
        hi[a:a + n] = torch.clamp(r + 1, min=a + p)
        a += n
    return lo, hi


def heads(t, n, d):
    return t.double().view(t.shape[0], n, d).transpose(0, 1)


def attention(T, nq, nkv, d, cap, lo, hi, qkv, half_step, dout=None, o_in=None, lse_in=None):
    """{"o", "lse", "dq", "dk", "dv"} as (value, bound), [heads, T, d] and lse [nq, T]; the backward pass from the given o and lse.  Masked entries never enter."""
    g, sc, u = nq // nkv, 1.0 / math.sqrt(d), half_step
    q = heads(qkv[:, :nq * d], nq, d)
    k = heads(qkv[:, nq * d:(nq + nkv) * d], nkv, d).repeat_interleave(g, 0)
    v = heads(qkv[:, (nq + nkv) * d:], nkv, d).repeat_interleave(g, 0)
    j = torch.arange(T)
    seen = (j[None, :] >= lo[:, None]) & (j[None, :] < hi[:, None])
    live = hi > lo

    def product(a, b):  # sum over the seen entries alone: zeros times infinities are left out
        return torch.matmul(a, torch.nan_to_num(b, nan=0.0, posinf=0.0, neginf=0.0))

    x = torch.matmul(q, k.transpose(1, 2)) * sc
    xa = torch.matmul(q.abs(), k.abs().transpose(1, 2)) * sc
    slope = torch.ones_like(x)
    y = x
    if cap:
        t = torch.tanh(x / cap)
        y, slope = cap * t, 1 - t * t
    y = y.masked_fill(~seen, -math.inf)
    top = torch.where(live, y.amax(2), torch.zeros(()).double())
    e = torch.exp(y - top[:, :, None])
    total = e.sum(2)
    lse = top + torch.log(torch.where(live, total, torch.ones(()).double()))
    n = (hi - lo).clamp(min=1).double()[None, :, None]

    def dy_of(ref):  # error of a probability's exponent
        return (((d + 8) * W * xa + 16 * W * cap + 4 * W * (x.abs() + ref.abs()[:, :, None])).masked_fill(~seen, 0.0)) + 2 ** -22

    out = {}
    if dout is None:
        p = torch.where(seen, e / torch.where(live, total, torch.ones(()).double())[:, :, None], torch.zeros(()).double())
        o = product(p, v)
        dp = dy_of(lse)
        rel = dp.amax(2, keepdim=True) * 2 + 2 * n * W + u
        oa = product(p, v.abs())
        out["o"] = (o, rel * oa + 1.01 * u * o.abs() + 1e-30)
        out["lse"] = (lse, dp.amax(2) + (n[:, :, 0] + 8) * W + 4 * W * lse.abs())
        return out
    do = heads(dout, nq, d)
    oi = heads(o_in, nq, d)
    L = lse_in.double()
    p = torch.where(seen, torch.exp(torch.where(seen, y, torch.zeros(()).double()) - L[:, :, None]), torch.zeros(()).double())
    delta = (do * oi).sum(2, keepdim=True)
    deltaa = (do * oi).abs().sum(2, keepdim=True)
    dp = torch.matmul(do, v.transpose(1, 2))
    dpa = torch.matmul(do.abs(), v.abs().transpose(1, 2))
    ds = torch.where(seen, p * (dp - delta) * slope, torch.zeros(()).double())
    pe = dy_of(L) * 2
    dse = torch.where(seen, (pe + u + 8 * W) * ds.abs() + p * ((d + 8) * W * (dpa + deltaa)) + p * (dp - delta).abs() * (32 * W if cap else 0.0), torch.zeros(()).double())

    def group(t):
        return t.view(nkv, g, T, d).sum(1)

    nk = seen.sum(0).clamp(min=1).double()[None, :, None] * g
    dq, dqe = product(ds, k) * sc, (product(dse, k.abs()) + 2 * n * W * product(ds.abs(), k.abs())) * sc
    dk = group(product(ds.transpose(1, 2), q)) * sc
    dke = (group(product(dse.transpose(1, 2), q.abs())) + 2 * nk * W * group(product(ds.abs().transpose(1, 2), q.abs()))) * sc
    dv = group(product(p.transpose(1, 2), do))
    dve = group(product(((pe + u) * p).transpose(1, 2), do.abs())) + 2 * nk * W * group(product(p.transpose(1, 2), do.abs()))
    for name, val, err in (("dq", dq, dqe), ("dk", dk, dke), ("dv", dv, dve)):
        out[name] = (val, err + 1.01 * u * val.abs() + 1e-30)
    return out
