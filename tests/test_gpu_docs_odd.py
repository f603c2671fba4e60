"""Infinities and NaNs in packed documents: those that a row sees and those it does not, in the same tiles.  A result is what the formulas give over exactly what is seen, infinities
with their sign, unless a row has no finite result at all; and it costs no more than a second walk over the tiles."""
import math

import pytest
import torch

import docs_ref as R
from test_gpu_docs_attn import Packed

pytestmark = pytest.mark.gpu
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def over_what_is_seen(p, o_in=None, lse_in=None):
    """o, lse, and from given o and lse delta, dq, dk, dv, [T, heads, d], a row at a time over its keys alone: float64 products of what is seen, whatever it is."""
    T, nq, nkv, d, cap, sc = p.T, p.nq, p.nkv, p.d, p.cap, 1.0 / math.sqrt(p.d)
    x = p.qkv.double().view(T, nq + 2 * nkv, d)
    q, k, v = x[:, :nq], x[:, nq:nq + nkv], x[:, nq + nkv:]
    do = p.dout.double().view(T, nq, d)
    o, lse = torch.zeros((T, nq, d)).double(), torch.zeros((T, nq)).double()
    dq, dk, dv = torch.zeros((T, nq, d)).double(), torch.zeros((T, nkv, d)).double(), torch.zeros((T, nkv, d)).double()
    for i in range(T):
        lo, hi = int(p.lo[i]), int(p.hi[i])
        for h in range(nq) if hi > lo else ():
            K, V = k[lo:hi, h // (nq // nkv)], v[lo:hi, h // (nq // nkv)]
            y = (K * q[i, h]).sum(1) * sc
            slope = torch.ones_like(y)
            if cap:
                t = torch.tanh(y / cap)
                y, slope = cap * t, 1 - t * t
            if o_in is None:
                lse[i, h] = torch.logsumexp(y, 0)
                o[i, h] = (torch.exp(y - lse[i, h])[:, None] * V).sum(0)
                continue
            P = torch.exp(y - float(lse_in[h, i]))
            delta = (do[i, h] * o_in[i, h]).sum()
            ds = P * ((V * do[i, h]).sum(1) - delta) * slope
            dq[i, h] = (ds[:, None] * K).sum(0) * sc
            dk[lo:hi, h // (nq // nkv)] += ds[:, None] * q[i, h] * sc
            dv[lo:hi, h // (nq // nkv)] += P[:, None] * do[i, h]
    return (o, lse) if o_in is None else (dq, dk, dv)


def same(got, want, size, what, rows, any_kind):
    """Infinities and NaNs as wanted (in rows of any_kind: as good as the other), finite numbers 2 % of `size` off at most: probabilities, their gradients and the results round to 2^-8
    each, relatively, and the sums' terms are no larger than a few times `size`."""
    got, want = got.double().cpu()[rows], want[rows]
    finite = torch.isfinite(want)
    kinds = torch.where(torch.isnan(want), torch.isnan(got), got == want) | any_kind[rows].view(-1, *([1] * (want.dim() - 1))) & ~torch.isfinite(got)
    near = (got - want).abs() <= 0.02 * size
    bad = ~torch.where(finite, near, kinds)
    assert not bad.any(), (what, int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][0].item(), want[bad][0].item())


@pytest.mark.parametrize("dtype,d,nq,nkv,lengths", [("bf16", 128, 2, 1, [70, 90, 30]), ("bf16", 64, 2, 2, [70, 90, 30]), ("bf16", 128, 1, 1, [700, 200]), ("bf16", 64, 1, 1, [900, 40]),
                                                    ("f32", 64, 2, 1, [70, 90, 30]), ("f32", 24, 1, 1, [70, 90, 30]), ("f32", 256, 1, 1, [70, 90, 30])])
@pytest.mark.parametrize("cap", [0.0, 50.0])
@pytest.mark.parametrize("where", ["v", "k", "dout"])
def test_single_elements(dh, dtype, d, nq, nkv, lengths, cap, where):
    """One element of the first document's middle row is an infinity, which later rows see in that column; beside it a row of NaNs at the document's end, which the rows before do not see, and
    the second document is NaNs altogether."""
    p = Packed(dh, dtype, T=sum(lengths) + 3, nq=nq, nkv=nkv, d=d, lengths=lengths, first=2, cap=cap, seed=31)
    a, mid = 2 + lengths[0], 2 + lengths[0] - 25
    kc, vc = nq * d, (nq + nkv) * d
    p.qkv[:a, :nq * d] *= 0.2  # no probability falls below what the kernels hold
    if where == "k":  # against queries of one the key's score is minus infinity: no weight (capped: of a slope of 0), but 0 times infinity in dq
        p.qkv[:, 5:nq * d:d] = 1.0
        p.qkv[mid, kc + 5] = -INF
    elif where == "v":
        p.qkv[mid, vc + 7] = INF
        p.qkv[mid + 3, vc + 9] = -INF
    else:
        p.dout[mid, 11] = INF
    for t in (p.qkv, p.dout):
        t[a - 1] = NAN
        t[a:a + lengths[1]] = NAN
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    o_in, lse_in = p.o.cpu().double().view(p.T, nq, d), p.lse.cpu().double()
    o, lse = over_what_is_seen(p)
    rows = p.live.clone()
    rows[a:a + lengths[1]] = False
    none = torch.zeros(p.T, dtype=torch.bool)
    same(p.o.view(p.T, nq, d), o, 4.0, "o", rows, none)
    same(p.lse.t(), lse, 1.0, "lse", rows, none)
    dq, dk, dv = over_what_is_seen(p, o_in, lse_in)
    got = p.dqkv.view(p.T, nq + 2 * nkv, d)
    # dq of a row whose delta is no number, dk of keys that see such a row, and everything of keys that see the row of NaNs: none of it is finite
    odd = ~torch.isfinite((p.dout.double().view(p.T, nq, d) * o_in).sum(2)).all(1)
    seen_odd = torch.tensor([bool(odd[j:a].any()) if j < a else False for j in range(p.T)])
    same(got[:, :nq], dq, 40.0, "dq", rows, odd)
    same(got[:, nq:nq + nkv], dk, 40.0, "dk", rows, seen_odd)
    same(got[:, nq + nkv:], dv, 40.0, "dv", rows, torch.arange(p.T) < a)


@pytest.mark.parametrize("d,cap", [(128, 0.0), (128, 30.0), (64, 0.0), (64, 30.0)])
def test_infinities_of_one_column_stay_there(dh, d, cap):
    """As above without NaNs that a row of the first document sees: dv holds infinities in one column and numbers in the others."""
    p = Packed(dh, "bf16", T=200, nq=1, nkv=1, d=d, lengths=[100, 90], first=0, cap=cap, seed=32)
    p.qkv[:100, :d] *= 0.2
    p.dout[60, 11] = INF
    for t in (p.qkv, p.dout):
        t[100:190] = NAN
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    dv = p.dqkv[:100, 2 * d:].float().cpu()
    other = torch.arange(d) != 11
    assert bool((dv[:61, 11] == INF).all()) and bool(torch.isfinite(dv[61:]).all()) and bool(torch.isfinite(dv[:61, other]).all())
    clean = Packed(dh, "bf16", T=200, nq=1, nkv=1, d=d, lengths=[100, 90], first=0, cap=cap, seed=32)
    clean.qkv[:100, :d] *= 0.2
    r = clean.ref(dout=clean.dout, o_in=torch.nan_to_num(p.o.cpu()), lse_in=torch.nan_to_num(p.lse.cpu()))["dv"]
    assert bool(((dv[:, other].double() - r[0][0, :100][:, other]).abs() <= r[1][0, :100][:, other]).all())
    dq, dk = p.dqkv[:100, :d].float().cpu(), p.dqkv[:100, d:2 * d].float().cpu()
    assert bool(torch.isfinite(dq[torch.arange(100) != 60]).all()) and not bool(torch.isfinite(dq[60]).any()) and bool(torch.isfinite(dk[61:]).all())


@pytest.mark.parametrize("d,cap", [(128, 0.0), (128, 30.0), (64, 0.0), (64, 30.0)])
def test_products_beyond_float32_that_are_not_seen(dh, d, cap):
    """Values of 1e30 in one document and gradients of 1e20 in its neighbour: their products, which nobody sees, pass float32's range."""
    def poison(qkv, dout):
        qkv[50:120, 2 * d + d:] *= 1e30
        dout[:50] *= 1e20
        dout[120:150] *= 1e20

    Packed(dh, "bf16", T=150, nq=2, nkv=1, d=d, lengths=[50, 70, 30], cap=cap, seed=33).run(poison)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("which", ["k", "v", "q"])
def test_a_nan_that_is_seen_arrives(dh, dtype, d, which):
    """One row's keys, values or queries are NaNs altogether: rows that see it hold NaNs (lse with a key or a query), the others none."""
    p = Packed(dh, dtype, T=170, nq=1, nkv=1, d=d, lengths=[70, 90], first=2, seed=35)
    p.qkv[47, {"q": slice(0, d), "k": slice(d, 2 * d), "v": slice(2 * d, 3 * d)}[which]] = NAN
    p.qkv_d = p.qkv.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    torch.cuda.synchronize()
    r = torch.arange(p.T)
    sees = r == 47 if which == "q" else (r >= 47) & (r < 72)
    o, lse = p.o.float().cpu(), p.lse.cpu()[0]
    assert bool(torch.isnan(o[sees]).all()) and bool(torch.isfinite(o[~sees]).all())
    assert torch.equal(torch.isnan(lse), sees if which != "v" else torch.zeros_like(sees))


@pytest.mark.parametrize("d,cap", [(128, 0.0), (128, 30.0), (64, 0.0), (64, 30.0)])
def test_a_row_without_weight(dh, d, cap):
    """lse of plus infinity, as a caller may pass for a row that is to count for nothing: its dq is zero and it adds nothing to dk and dv, beside a document of NaNs in the same tile."""
    p = Packed(dh, "bf16", T=200, nq=1, nkv=1, d=d, lengths=[100, 90], first=0, cap=cap, seed=36)
    for t in (p.qkv, p.dout):
        t[100:190] = NAN
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.lse[:, 80] = INF
    p.backward()
    torch.cuda.synchronize()
    got = p.dqkv[:100].float().cpu()
    clean = Packed(dh, "bf16", T=200, nq=1, nkv=1, d=d, lengths=[100, 90], first=0, cap=cap, seed=36)
    clean.dout[80] = 0.0  # the same as a row of no gradient, whose delta is zero
    o = torch.nan_to_num(p.o.cpu())
    lse = torch.nan_to_num(p.lse.cpu(), posinf=0.0)
    lse[:, 80] = 1e4  # exp(score - lse) = 0
    r = clean.ref(dout=clean.dout, o_in=o, lse_in=lse)
    assert not bool(got[80, :d].any())
    for i, name in enumerate(("dq", "dk", "dv")):
        val, err = (t[0, :100] for t in r[name])
        assert bool(((got[:, i * d:(i + 1) * d].double() - val).abs() <= err).all()), name


def microseconds(f):
    f()
    torch.cuda.synchronize()
    best = INF
    for _ in range(3):
        s, e = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        s.record()
        f()
        e.record()
        e.synchronize()
        best = min(best, s.elapsed_time(e) * 1e3)
    return best


@pytest.mark.parametrize("d,cap,nq,nkv", [(128, 0.0, 4, 1), (64, 0.0, 8, 2), (128, 50.0, 4, 2)])
def test_what_they_cost(dh, d, cap, nq, nkv):
    """One document of 8192 rows.  At most a wave's tiles are walked twice, in a slower form: less than 16 times the time without, where one row after the other took 100 times as long."""
    T, h = 8192, 6000
    docs = Packed(dh, "bf16", T=T, nq=nq, nkv=nkv, d=d, lengths=[T], cap=cap, seed=34)
    docs.qkv_d, docs.dout_d = docs.qkv.cuda(), docs.dout.cuda()
    docs.buffers()
    dh.dh_docs_plan(docs.docs)
    fwd, bwd = microseconds(docs.forward), microseconds(docs.backward)
    vc = (nq + nkv) * d
    q, g = docs.qkv_d, docs.dout_d
    for name, write in [("a token", lambda: q[h].fill_(NAN)), ("everything from a token on", lambda: q[h:].fill_(NAN)), ("the first token", lambda: q[0].fill_(NAN)),
                        ("values from a token on", lambda: q[h:, vc:].fill_(NAN)), ("a value", lambda: q[h, vc:].fill_(INF)), ("all gradients", lambda: g.fill_(NAN)),
                        ("infinite gradients", lambda: g.fill_(INF)), ("a gradient", lambda: g[h].fill_(NAN))]:
        q.copy_(docs.qkv)
        g.copy_(docs.dout)
        write()
        f, b = microseconds(docs.forward), microseconds(docs.backward)
        assert f <= 16 * fwd and b <= 16 * bwd, (name, f, fwd, b, bwd)
