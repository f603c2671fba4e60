"""Attention inside packed documents in forms that its other tests do not take: every launch form of the backward pass, tables for other sizes, more rows than one launch counts."""
import os
import re

import pytest
import torch

import docs_ref as R
from test_gpu_docs_attn import MARK, Packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    yield dhelix
    torch.cuda.empty_cache()


def prepared(p):
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    return p


@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 2, 1, 128), ("bf16", 2, 2, 64), ("bf16", 64, 16, 128), ("f32", 2, 1, 64), ("f32", 2, 1, 256)])
def test_delta_of_rows_of_no_document_stays(dh, dtype, nq, nkv, d):
    """In one launch and in two; delta of the others is rowsum(dout o), a sum of d products."""
    p = prepared(Packed(dh, dtype, T=2100 if nq == 64 else 200, nq=nq, nkv=nkv, d=d, lengths=[30, 0, 70, 50], first=9, seed=21))
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    delta = p.delta.cpu()
    assert bool((delta[:, ~p.live] == MARK).all())
    do, o = (t.double().cpu().view(p.T, nq, d).transpose(0, 1) for t in (p.dout, p.o))
    assert bool((((delta.double() - (do * o).sum(2)).abs() <= (d + 8) * R.W * (do * o).abs().sum(2))[:, p.live]).all())


@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 4, 2, 64), ("bf16", 4, 2, 128), ("bf16", 64, 32, 128), ("f32", 4, 2, 64), ("f32", 4, 2, 256)])
@pytest.mark.parametrize("other", ["heads", "rows"])
def test_a_table_for_other_sizes_changes_nothing(dh, dtype, nq, nkv, d, other):
    """Both passes, in one launch and in two, with a table for other heads or other rows in a buffer that holds either: every output is as it was."""
    T = 1500 if nq == 64 else 300
    p = Packed(dh, dtype, T=T, nq=nq, nkv=nkv, d=d, lengths=[T], seed=22)
    p.table = torch.zeros(max(dh.dh_docs_table_bytes(T, nq, k) for k in (1, nkv, nq)), dtype=torch.uint8, device="cuda")
    made = dh.docs(T if other == "heads" else T - 64, 1, nq, 1 if other == "heads" else nkv, p.start, None, None, p.table)
    p.docs = dh.docs(T, 1, nq, nkv, p.start, None, None, p.table)
    prepared(p)
    dh.dh_docs_plan(made)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    for t in (p.o, p.lse, p.dqkv, p.delta):
        assert bool((t == MARK).all())


@pytest.mark.parametrize("first", [2 ** 26 - 60, 2 ** 27 - 100])
def test_more_rows_than_a_launch_counts(dh, first):
    """Float32, 2^27 + 200 rows: a block of 512 threads for every 16 rows passes 32 bits.  Two documents across the border of two launches."""
    T, S, d, lengths, base = 2 ** 27 + 200, 256, 8, [100, 70], first - 16
    g = torch.Generator().manual_seed(23)
    qkv, dout = torch.randn((S, 3 * d), generator=g), torch.randn((S, d), generator=g)
    lo, hi = R.tables(S, lengths, None, 16)
    rows, live = slice(base, base + S), slice(16, 16 + sum(lengths))
    Q, D, O, DQ = (torch.empty((T, n), device="cuda") for n in (3 * d, d, d, 3 * d))
    Q[rows], D[rows] = qkv.cuda(), dout.cuda()
    lse, delta = torch.full((1, T), MARK, device="cuda"), torch.full((1, T), MARK, device="cuda")
    for t in (O, DQ):
        t.fill_(MARK)
    start = torch.tensor([first, first + 100, first + 170], dtype=torch.int32, device="cuda")
    table = torch.empty(dh.dh_docs_table_bytes(T, 1, 1), dtype=torch.uint8, device="cuda")
    docs = dh.docs(T, 2, 1, 1, start, None, None, table)
    dh.dh_docs_plan(docs)
    dh.dh_attn_docs_fwd(dh.DH_F32, docs, d, 0.0, Q, O, lse)
    dh.dh_attn_docs_bwd(dh.DH_F32, docs, d, 0.0, Q, O, D, lse, DQ, delta)
    torch.cuda.synchronize()
    o, l, dq = O[rows].cpu(), lse[:, rows].cpu(), DQ[rows].cpu()
    u = 2.0 ** -24
    r = R.attention(S, 1, 1, d, 0.0, lo, hi, qkv, u)
    b = R.attention(S, 1, 1, d, 0.0, lo, hi, qkv, u, dout=dout, o_in=o, lse_in=l)
    for got, pair in ((o, r["o"]), (dq[:, :d], b["dq"]), (dq[:, d:2 * d], b["dk"]), (dq[:, 2 * d:], b["dv"]), (l.t(), [t[:, :, None] for t in r["lse"]])):
        val, err = (t.transpose(0, 1).reshape(S, -1)[live] for t in pair)
        assert bool(((got[live].double() - val).abs() <= err).all())
    for t, n in ((O, d), (DQ, 3 * d), (lse.view(T, 1), 1), (delta.view(T, 1), 1)):
        others = sum(int((part != MARK).sum()) for part in t.split(1 << 24))
        assert others <= 170 * n and int((t[first:first + 170] != MARK).sum()) == others  # nothing outside the documents changed


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 256), ("f32", 24)])
@pytest.mark.parametrize("length", [40, 900])
def test_rows_whose_scores_are_all_minus_infinity(dh, dtype, d, length):
    """The second document's keys are minus infinities against queries of ones: lse is minus infinity, o a NaN, whatever the type and whether rows are cut.  With a finite score beside
    them (the last key) a row has that key's value alone."""
    T = length + 60
    p = Packed(dh, dtype, T=T, nq=2, nkv=1, d=d, lengths=[50, length], seed=24)
    p.qkv[50:, 2 * d] = float("-inf")  # one element of every key
    p.qkv[:, :2 * d] = 1.0
    p.qkv[49 + length, 2 * d] = 0.5
    prepared(p)
    dh.dh_docs_plan(p.docs)
    p.forward()
    torch.cuda.synchronize()
    o, lse = p.o.cpu().view(T, 2, d).float(), p.lse.cpu()
    assert bool((lse[:, 50:49 + length] == float("-inf")).all()) and bool(torch.isnan(o[50:49 + length]).all())
    last = 49 + length
    k, v = p.qkv[last, 2 * d:3 * d].double(), p.qkv[last, 3 * d:].float()
    x, size = float(k.sum()) / d ** 0.5, float(k.abs().sum()) / d ** 0.5
    assert bool(((lse[:, last].double() - x).abs() <= (d + 16) * R.W * size + 2 ** -22).all()) and torch.equal(o[last], v.expand(2, d))
    assert bool(torch.isfinite(o[:50]).all()) and bool(torch.isfinite(lse[:, :50]).all())


@pytest.mark.parametrize("T,nq,nkv,d", [(17000, 24, 8, 64), (10000, 12, 4, 128)])
@pytest.mark.parametrize("cap", [0.0, 30.0])
def test_two_launches_with_cut_blocks(dh, T, nq, nkv, d, cap):
    """More blocks than the backward pass takes in one launch, so that dQ leaves the statistics for dK and dV, and a document of 3000 rows among short ones, whose blocks of queries and of keys are cut.
    Checked: that document's first and last group of heads, and the first and the last short document's."""
    from paper_2411_15871_amd import build as B
    table_h, attn_h = (open(os.path.join(B.CSRC, f)).read() for f in ("docs.h", "attn_docs_bf16.h"))
    assert "D == 128 ? DOCS_ONE_128 : 4 * DOCS_ONE_64)) {" in attn_h  # the limits that this test is to pass
    limit = {n: int(re.search(r"#define DOCS_ONE_%d (\d+)" % n, table_h).group(1)) for n in (64, 128)}
    assert (T + 127) // 128 * (nq + nkv) > (limit[128] if d == 128 else 4 * limit[64])
    short = (T - 3000 - 90) // 100
    lengths = [90] + [3000] + [100] * short
    p = prepared(Packed(dh, "bf16", T=T, nq=nq, nkv=nkv, d=d, lengths=lengths, first=0, cap=cap, seed=25))
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    cut = p.table[:64].view(torch.int32).cpu()[6::2].tolist()  # forward, dQ of heads of 128 and of 64, dK and dV
    assert cut[0] > 0 and cut[2 if d == 64 else 1] > 0 and cut[4 if d == 64 else 3] > 0
    o, lse, dqkv, delta = p.o.cpu(), p.lse.cpu(), p.dqkv.cpu(), p.delta.cpu()
    assert bool(torch.isfinite(dqkv[p.live].float()).all()) and bool((dqkv[~p.live] == MARK).all()) and bool((delta[:, ~p.live] == MARK).all())
    grp = nq // nkv
    for a, n, groups in ((90, 3000, (0, nkv - 1)), (0, 90, range(nkv)), (3090, 100, range(nkv)), (3090 + 100 * (short - 1), 100, range(nkv))):
        rows, lo = slice(a, a + n), torch.zeros(n, dtype=torch.long)
        for g in groups:
            hs = slice(g * grp, (g + 1) * grp)
            x = [p.qkv[rows, i * d:j * d] for i, j in ((g * grp, (g + 1) * grp), (nq + g, nq + g + 1), (nq + nkv + g, nq + nkv + g + 1))]
            args = (n, grp, 1, d, cap, lo, torch.arange(1, n + 1), torch.cat(x, 1), p.u)
            fwd = R.attention(*args)
            bwd = R.attention(*args, dout=p.dout[rows, g * grp * d:(g + 1) * grp * d], o_in=o[rows, g * grp * d:(g + 1) * grp * d], lse_in=lse[hs, rows])
            got = {"o": o[rows, g * grp * d:(g + 1) * grp * d], "dq": dqkv[rows, g * grp * d:(g + 1) * grp * d], "dk": dqkv[rows, (nq + g) * d:(nq + g + 1) * d],
                   "dv": dqkv[rows, (nq + nkv + g) * d:(nq + nkv + g + 1) * d]}
            for name, t in got.items():
                val, err = (z.transpose(0, 1).reshape(n, -1) for z in (fwd if name == "o" else bwd)[name])
                assert bool(((t.double() - val).abs() <= err).all()), (name, a, g)
            assert bool(((lse[hs, rows].double() - fwd["lse"][0]).abs() <= fwd["lse"][1]).all()), (a, g)
