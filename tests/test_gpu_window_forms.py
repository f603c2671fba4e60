"""Window attention at sizes that take its other launches: two of the backward pass in both types, walks over keys cut into parts, more blocks of sinks than are cut, more blocks of a row than
one axis of a launch has; with infinities and NaNs before a row's window in each (tests/mixers_ref.py holds the formulas and the bounds)."""
import math

import pytest
import torch

import mixers_ref as R
from test_gpu_window_attn import BF, F, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def check_each(c, hurt=None, grad=None):
    """Every sequence by itself.  hurt: rows of the first that see what is not finite; grad: and those whose gradient is not.  Returns how many of its rows and keys were compared."""
    seen = R.seen_by(1, c.seq, c.window, c.sinks)
    a, b, count = c.nq * c.d, (c.nq + c.nkv) * c.d, None
    for s in range(c.batch):
        at = slice(s * c.seq, (s + 1) * c.seq)
        fine = (None, None, None)
        if s == 0 and hurt is not None:
            fine = (~hurt, ~(hurt | grad), ~seen[hurt | grad].any(0))
            count = [int(f.sum()) for f in fine]
        rows, rows_g, keys = (None if f is None else f[:, None] for f in fine)
        o, lse = c.o[at], c.lse[:, at]
        fwd = R.attention(seen, c.nq, c.nkv, c.d, c.qkv[at])
        R.check(o, fwd["o"], "o of %d" % s, rows)
        R.check(lse, fwd["lse"], "lse of %d" % s, None if rows is None else rows[:, 0][None, :])
        bwd = R.attention(seen, c.nq, c.nkv, c.d, c.qkv[at], c.dout[at], o.cpu(), lse.cpu())
        R.check(c.dqkv[at, :a], bwd["dq"], "dq of %d" % s, rows_g)
        R.check(c.dqkv[at, a:b], bwd["dk"], "dk of %d" % s, keys)
        R.check(c.dqkv[at, b:], bwd["dv"], "dv of %d" % s, keys)
    return count


FORMS = [(F, 8, 500, 90, 5, 8, 2, 32), (F, 5, 520, 200, 130, 8, 8, 40), (F, 3, 700, 1000, 0, 16, 4, 128),  # more than 2048 blocks of 16 rows
         (BF, 6, 700, 200, 4, 32, 8, 64), (BF, 7, 650, 90, 130, 32, 8, 64),                                  # more than 1280 blocks of 128
         (BF, 3, 700, 200, 4, 32, 8, 128), (BF, 3, 650, 90, 130, 32, 8, 128),                                # more than 512
         (BF, 1, 1500, 1300, 70, 2, 1, 64), (BF, 1, 1500, 1300, 70, 2, 1, 128), (BF, 2, 1201, 2000, 0, 1, 1, 64),  # parts
         (BF, 1, 1500, 50, 1100, 2, 2, 64), (BF, 1, 1500, 50, 1100, 2, 2, 128),                              # nine blocks of sinks
         (BF, 1, 1500, 300, 1100, 4, 1, 64), (BF, 1, 1500, 300, 1100, 4, 1, 128)]                            # beside other blocks that are cut


@pytest.mark.parametrize("tt,batch,seq,window,sinks,nq,nkv,d", FORMS)
def test_both_passes(dh, tt, batch, seq, window, sinks, nq, nkv, d):
    c = Case(dh, tt, batch, seq, window, sinks, nq, nkv, d, seed=seq).upload()
    c.forward()
    c.backward()
    check_each(c)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("which", ["v", "k", "dout"])
@pytest.mark.parametrize("tt,batch,seq,window,sinks,nq,nkv,d", [(BF, 1, 1500, 1300, 70, 2, 1, 64), (BF, 1, 1500, 1300, 70, 2, 1, 128), (BF, 1, 1500, 300, 40, 4, 2, 64),
                                                                (BF, 1, 1500, 300, 40, 4, 2, 128), (BF, 6, 700, 200, 0, 32, 8, 64), (BF, 3, 700, 200, 0, 32, 8, 128),
                                                                (F, 5, 520, 200, 0, 8, 8, 40)])
def test_what_lies_before_a_window(dh, tt, batch, seq, window, sinks, nq, nkv, d, which, bad):
    """Two tokens that rows of the window's length see and those behind these do not, in tiles that both walk."""
    c = Case(dh, tt, batch, seq, window, sinks, nq, nkv, d, seed=3)
    a, b, at = nq * d, (nq + nkv) * d, torch.tensor([100, 131])
    hurt, grad = torch.zeros(seq, dtype=torch.bool), torch.zeros(seq, dtype=torch.bool)
    if which == "dout":
        c.dout[at, 2::5] = bad
        grad[at] = True
    else:
        first = b if which == "v" else a
        c.qkv[at, first + 3:first + nkv * d:7] = bad
        hurt = R.seen_by(1, seq, window, sinks)[:, at].any(1)
    c.upload()
    c.forward()
    c.backward()
    rows, rows_g, keys = check_each(c, hurt, grad)
    assert rows_g >= 100 + (seq - 131 - window) and keys >= seq - 131 - window > 0
    assert not torch.isfinite((c.dqkv if which == "dout" else c.o)[100].float()).all()


@pytest.mark.parametrize("d", [64, 128])
def test_more_blocks_than_an_axis(dh, d):
    """2^22 rows and some: the last blocks lie behind the first 32768 of a row, and the sinks' gradients gather from all."""
    seq, window, sinks, tail = 2 ** 22 + 777, 100, 3, 1200
    g = torch.Generator(device="cuda").manual_seed(1)
    draw = lambda n: torch.randn((seq, n), generator=g, device="cuda", dtype=torch.float32).to(BF)  # noqa: E731
    qkv, dout = draw(3 * d), draw(d)
    args = (dh.DH_BF16, 1, seq, window, sinks, 1, 1, d)
    o, lse, dqkv, delta = torch.full_like(dout, 7.0), torch.full((1, seq), 7.0, device="cuda"), torch.full_like(qkv, 7.0), torch.full((1, seq), 7.0, device="cuda")
    n = max(16, dh.dh_attn_window_fwd_workspace_bytes(*args), dh.dh_attn_window_bwd_workspace_bytes(*args))
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")
    dh.dh_attn_window_fwd(*args, qkv, o, lse, ws, n)
    dh.dh_attn_window_bwd(*args, qkv, o, dout, lse, dqkv, delta, ws, n)
    # the last rows, with the sinks in front; those whose window begins before the tail do not count
    cut = lambda t: torch.cat([t[:sinks], t[seq - tail:]]).cpu()  # noqa: E731
    m = sinks + tail
    i = torch.arange(m)
    seen = (i[None, :] <= i[:, None]) & ((i[None, :] < sinks) | (i[None, :] > i[:, None] - window))
    fine = i >= sinks + window
    q, do, lo = cut(qkv), cut(dout), cut(lse.T).T.contiguous()
    fwd = R.attention(seen, 1, 1, d, q)
    R.check(cut(o), fwd["o"], "o", fine[:, None])
    R.check(lo, fwd["lse"], "lse", fine[None, :])
    bwd = R.attention(seen, 1, 1, d, q, do, cut(o), lo)
    for k, name in enumerate(("dq", "dk", "dv")):
        R.check(cut(dqkv)[:, k * d:(k + 1) * d], bwd[name], name, fine[:, None])
    # the sinks' gradients, in float64 over all rows: probabilities and their gradients round to 2^-8, and seq + 2 terms are added in float32
    x = qkv.double()
    k, v, w = x[:sinks, d:2 * d], x[:sinks, 2 * d:], dout.double()
    sees = torch.arange(seq, device="cuda")[:, None] >= torch.arange(sinks, device="cuda")[None, :]
    p = torch.where(sees, torch.exp(x[:, :d] @ k.T / math.sqrt(d) - lse[0].double()[:, None]), torch.zeros((), dtype=torch.float64, device="cuda"))
    ds = p * (w @ v.T - (w * o.double()).sum(1, keepdim=True)) / math.sqrt(d)
    for name, got, weights, of in (("dk", dqkv[:sinks, d:2 * d], ds, x[:, :d]), ("dv", dqkv[:sinks, 2 * d:], p, w)):
        val, size = weights.T @ of, weights.abs().T @ of.abs()
        R.check(got, (val.cpu(), (2.0 ** -8 * 1.1 * size + (seq + 2) * R.W * size + 1.01 * 2.0 ** -8 * val.abs()).cpu()), "sinks' " + name)
