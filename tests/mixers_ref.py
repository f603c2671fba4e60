"""Window attention, linear attention and dropout from their formulas in float64, with a bound for each result of a kernel that rounds as described.

With u = half a step of the storage type (2^-8 for bfloat16, 2^-24 for float32) and w = 2^-24:

Attention: the kernel may round the probabilities and their gradients to the storage type before the products that consume them, keeps every sum in float32, and rounds its results once.
  a score of d products is off by at most (d + 8) w sum |q k| / sqrt(d), the exponent by that and 4 w (|score| + |lse|) more;  a probability by its exponent's error, relatively, and u;
  a sum over n terms adds n w of the terms' magnitudes.

Linear attention: with A the result's formula over magnitudes, a term of it passes at most three roundings to the storage type before it is added (a weighted score, a state that is read, a
row that is weighted on its way into a state within a piece of a row: u each), sums of at most n + d + d terms, and a power of lambda: lambda^m is off by at most (2 + |m log lambda|) 4 w, relatively,
where |m log lambda| e^-|m log lambda| <= 1/e, so 6 w A covers it, once for each of the pieces that a long row is cut into, of at least 64 rows.  States are float32 in both types: no u.
"""
import math

import torch

W = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def heads(t, n, d):
    return t.double().view(t.shape[0], n, d).transpose(0, 1)


def rows(t):
    """[heads, T, d] -> [T, heads * d]"""
    return t.transpose(0, 1).reshape(t.shape[1], -1)


def seen_by(batch, seq, window, sinks):
    """[T, T]: which keys each row sees."""
    T = batch * seq
    t = torch.arange(T)
    i, j, same = (t % max(seq, 1))[:, None], (t % max(seq, 1))[None, :], (t // max(seq, 1))[:, None] == (t // max(seq, 1))[None, :]
    return same & (j <= i) & ((j > i - window) | (j < sinks))


def finite(t):
    return torch.nan_to_num(t, nan=0.0, posinf=0.0, neginf=0.0)


def attention(seen, nq, nkv, d, qkv, dout=None, o_in=None, lse_in=None):
    """{"o", "lse"} or, with the backward pass' inputs, {"dq", "dk", "dv"}, as (value, bound): [T, heads * d], lse [nq, T].  What a row does not see never enters."""
    u, g, sc, T = half_step(qkv.dtype), nq // nkv, 1.0 / math.sqrt(d), qkv.shape[0]
    q = heads(qkv[:, :nq * d], nq, d)
    k = heads(qkv[:, nq * d:(nq + nkv) * d], nkv, d).repeat_interleave(g, 0)
    v = heads(qkv[:, (nq + nkv) * d:], nkv, d).repeat_interleave(g, 0)
    zero = torch.zeros((), dtype=torch.float64)
    n = seen.sum(1).clamp(min=1).double()[None, :, None]
    x = torch.matmul(q, k.transpose(1, 2)) * sc
    xa = torch.matmul(q.abs(), k.abs().transpose(1, 2)) * sc

    def exponent(ref):
        return torch.where(seen, (d + 8) * W * xa + 4 * W * (x.abs() + ref.abs()[:, :, None]), zero) + 2 ** -22

    if dout is None:
        y = x.masked_fill(~seen, -math.inf)
        lse = torch.logsumexp(y, 2)
        p = torch.where(seen, torch.exp(y - lse[:, :, None]), zero)
        off = exponent(lse)
        oa = torch.matmul(p, finite(v).abs())
        o = torch.matmul(p, finite(v))
        return {"o": (rows(o), rows((off.amax(2, keepdim=True) * 2 + 2 * n * W + u) * oa + 1.01 * u * o.abs() + 1e-30)),
                "lse": (lse, off.amax(2) + (n[:, :, 0] + 8) * W + 4 * W * lse.abs())}
    do, L = heads(dout, nq, d), lse_in.double()
    p = torch.where(seen, torch.exp(torch.where(seen, x, zero) - L[:, :, None]), zero)
    do_o = do * heads(o_in, nq, d)
    delta, deltaa = do_o.sum(2, keepdim=True), do_o.abs().sum(2, keepdim=True)
    dp, dpa = torch.matmul(do, v.transpose(1, 2)), torch.matmul(do.abs(), v.abs().transpose(1, 2))
    ds = torch.where(seen, p * (dp - delta), zero)
    pe = exponent(L) * 2
    dse = torch.where(seen, (pe + u + 8 * W) * ds.abs() + p * ((d + 8) * W * (dpa + deltaa)), zero)

    def group(t):
        return t.view(nkv, g, T, d).sum(1)

    def product(a, b):
        return torch.matmul(a, finite(b))

    nk = seen.sum(0).clamp(min=1).double()[None, :, None] * g
    out = {}
    for name, val, err in (
            ("dq", product(ds, k) * sc, (product(dse, k.abs()) + 2 * n * W * product(ds.abs(), k.abs())) * sc),
            ("dk", group(product(ds.transpose(1, 2), q)) * sc, (group(product(dse.transpose(1, 2), q.abs())) + 2 * nk * W * group(product(ds.abs().transpose(1, 2), q.abs()))) * sc),
            ("dv", group(product(p.transpose(1, 2), do)), group(product(((pe + u) * p).transpose(1, 2), do.abs())) + 2 * nk * W * group(product(p.transpose(1, 2), do.abs())))):
        out[name] = (rows(val), rows(err + 1.01 * u * val.abs() + 1e-30))
    return out


def _linear(batch, seq, nq, nkv, d, scale, lam, qkv, state, dout, dstate):
    """The recurrence and its gradient, token by token."""
    g = nq // nkv
    x = qkv.view(batch, seq, nq + 2 * nkv, d)
    q, k, v = x[:, :, :nq].reshape(batch, seq, nkv, g, d), x[:, :, nq:nq + nkv], x[:, :, nq + nkv:]
    do = None if dout is None else dout.view(batch, seq, nkv, g, d)
    f = lam[None, :, None, None]
    S, o, dq = state.clone(), torch.zeros_like(q), torch.zeros_like(q)
    for t in range(seq):
        S = torch.where(f == 0, torch.zeros_like(S), f * S) + k[:, t, :, :, None] * v[:, t, :, None, :]
        o[:, t] = scale * torch.matmul(q[:, t], S)
        if do is not None:
            dq[:, t] = scale * torch.matmul(do[:, t], S.transpose(2, 3))
    T = batch * seq
    if do is None:
        return {"o": o.reshape(T, nq * d), "state": S}
    R, dk, dv = dstate.clone(), torch.zeros_like(k), torch.zeros_like(v)
    for t in reversed(range(seq)):
        R = R + scale * torch.matmul(q[:, t].transpose(2, 3), do[:, t])
        dk[:, t] = torch.matmul(R, v[:, t, :, :, None])[..., 0]
        dv[:, t] = torch.matmul(R.transpose(2, 3), k[:, t, :, :, None])[..., 0]
        R = torch.where(f == 0, torch.zeros_like(R), f * R)
    return {"dq": dq.reshape(T, nq * d), "dk": dk.reshape(T, nkv * d), "dv": dv.reshape(T, nkv * d), "dstate": R}


def linear(batch, seq, nq, nkv, d, scale, log_decay, qkv, state=None, dout=None, dstate=None):
    """{"o", "state"} or {"dq", "dk", "dv", "dstate"} as (value, bound)."""
    u, lam = half_step(qkv.dtype), torch.exp(log_decay.double())
    zeros = torch.zeros((batch, nkv, d, d), dtype=torch.float64)
    args = [qkv.double(), zeros if state is None else state.double(), None if dout is None else dout.double(), zeros if dstate is None else dstate.double()]
    val = _linear(batch, seq, nq, nkv, d, scale, lam, *args)
    mag = _linear(batch, seq, nq, nkv, d, abs(scale), lam, *[None if a is None else a.abs() for a in args])
    sums = (seq * (nq // nkv) + 2 * d + 16 + 6 * (1 + seq // 64)) * W
    out = {}
    for name in val:
        if name in ("state", "dstate"):
            out[name] = (val[name], (sums + 2 * W) * mag[name] + 1e-30)
        else:
            out[name] = (val[name], (sums + 3 * u) * mag[name] + 1.01 * u * val[name].abs() + 1e-30)
    return out


def philox(counter, key):
    """Philox4x32-10 on whole numbers."""
    x, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * x[0], 0xCD9E8D57 * x[2]
        x = [(b >> 32) ^ x[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ x[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def keep_mask(T, H, p, key, step, site):
    key, step = key % 2 ** 64, step % 2 ** 64
    bits = []
    for v in range(T * H // 8):
        for w in philox([v & 0xFFFFFFFF, v >> 32, step & 0xFFFFFFFF, site], [key & 0xFFFFFFFF, key >> 32]):
            bits += [w & 0xFFFF, w >> 16]
    below = int(65536 * p + 0.5)
    return (torch.tensor(bits, dtype=torch.int64) >= below).view(T, H), (0.0 if below == 65536 else 65536.0 / (65536 - below))


def check(got, pair, what, where=None):
    """got against (value, bound); where: which elements count.  A NaN is wrong."""
    val, err = pair
    got = got.detach().double().cpu().reshape(val.shape)
    bad = ~((got - val).abs() <= err)
    if where is not None:
        bad &= where
    assert not bad.any(), "%s: %d of %d wrong, first at %s: %r, wanted %r +- %r" % (
        what, int(bad.sum()), bad.numel(), bad.nonzero()[0].tolist(), got[bad][0].item(), val[bad][0].item(), err[bad][0].item())
