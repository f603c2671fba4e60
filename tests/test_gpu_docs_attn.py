"""Attention inside packed documents through the C ABI, against float64 (tests/docs_ref.py holds the formulas and the bounds)."""
import numpy as np
import pytest
import torch

import docs_ref as R

pytestmark = pytest.mark.gpu
MARK = 7.0  # what rows of no document hold before and after


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


class Packed:
    def __init__(self, dh, dtype, T, nq, nkv, d, lengths, prefixes=None, first=0, cap=0.0, seed=1):
        self.dh, self.bf16, self.T, self.nq, self.nkv, self.d, self.cap = dh, dtype == "bf16", T, nq, nkv, d, cap
        self.dt = dh.DH_BF16 if self.bf16 else dh.DH_F32
        self.tt = torch.bfloat16 if self.bf16 else torch.float32
        self.u = 2.0 ** -8 if self.bf16 else 2.0 ** -24
        self.lo, self.hi = R.tables(T, lengths, prefixes, first)
        self.live = self.hi > self.lo
        g = torch.Generator().manual_seed(seed)
        self.qkv = torch.randn((T, (nq + 2 * nkv) * d), generator=g)
        self.qkv[:, :nq * d] *= 2.5
        self.qkv = self.qkv.to(self.tt)
        self.dout = torch.randn((T, nq * d), generator=g).to(self.tt)
        starts = np.concatenate([[first], first + np.cumsum(lengths)]).astype(np.int32)
        self.start = torch.from_numpy(starts).cuda()
        self.prefix = torch.tensor(prefixes, dtype=torch.int32, device="cuda") if prefixes else None
        self.pos = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        self.table = torch.full((max(16, dh.dh_docs_table_bytes(T, nq, nkv)),), 0x5a, dtype=torch.uint8, device="cuda")
        self.docs = dh.docs(T, len(lengths), nq, nkv, self.start, self.prefix, self.pos, self.table)

    def buffers(self):
        full = lambda shape, t: torch.full(shape, MARK, dtype=t, device="cuda")  # noqa: E731
        self.o, self.lse = full((self.T, self.nq * self.d), self.tt), full((self.nq, self.T), torch.float32)
        self.dqkv, self.delta = full(tuple(self.qkv.shape), self.tt), full((self.nq, self.T), torch.float32)
        f = self.dh.dh_attn_docs_fwd_workspace_bytes(self.dt, self.T, self.nq, self.nkv, self.d)
        b = self.dh.dh_attn_docs_bwd_workspace_bytes(self.dt, self.T, self.nq, self.nkv, self.d)
        self.wsb = max(f, b)
        self.ws = torch.full((max(self.wsb, 16),), 0xff, dtype=torch.uint8, device="cuda")  # NaNs

    def forward(self, stream=None):
        self.dh.dh_attn_docs_fwd(self.dt, self.docs, self.d, self.cap, self.qkv_d, self.o, self.lse, self.ws, self.wsb, stream)

    def backward(self, stream=None):
        self.dh.dh_attn_docs_bwd(self.dt, self.docs, self.d, self.cap, self.qkv_d, self.o, self.dout_d, self.lse, self.dqkv, self.delta, self.ws, self.wsb, stream)

    def ref(self, **kw):
        return R.attention(self.T, self.nq, self.nkv, self.d, self.cap, self.lo, self.hi, self.qkv, self.u, **kw)

    def check(self, got, pair, what, rows=None):
        """got [T, heads*d] against (value, bound) [heads, T, d]; rows of no document hold what they held."""
        T, rows = self.T, self.live if rows is None else rows
        val, err = (t.transpose(0, 1).reshape(T, -1) for t in pair)
        got = got.double().cpu()
        bad = ((got - val).abs() <= err).logical_not() & rows[:, None]  # a NaN is bad
        assert not bad.any(), "%s: %d bad, first at %s: %s, wanted %s +- %s" % (
            what, int(bad.sum()), bad.nonzero()[0].tolist(), got[bad][0].item(), val[bad][0].item(), err[bad][0].item())

    def run(self, poison=None, rows=None):
        """Forward and backward, checked; poison(qkv, dout): writes what must not spread beyond `rows`' complement."""
        if poison:
            poison(self.qkv, self.dout)
        self.qkv_d, self.dout_d = self.qkv.cuda(), self.dout.cuda()
        dead = ~self.live
        self.buffers()
        self.dh.dh_docs_plan(self.docs)
        self.forward()
        torch.cuda.synchronize()
        fwd = self.ref()
        live = self.live if rows is None else rows & self.live
        pos = torch.where(self.live, torch.arange(self.T) - self.lo, torch.zeros((), dtype=torch.long))
        assert torch.equal(self.pos.cpu().long(), pos)
        self.check(self.o, fwd["o"], "o", live)
        lse, err = fwd["lse"]
        assert bool((((self.lse.cpu().double() - lse).abs() <= err) | ~live[None, :]).all()), "lse"
        assert bool((self.o.cpu()[dead] == MARK).all()) and bool((self.lse.cpu()[:, dead] == MARK).all())
        # the backward pass gets what the forward pass left
        self.backward()
        torch.cuda.synchronize()
        o_in, lse_in = self.o.cpu(), self.lse.cpu()
        r = self.ref(dout=self.dout, o_in=o_in, lse_in=lse_in)
        nq, nkv, d = self.nq, self.nkv, self.d
        self.check(self.dqkv[:, :nq * d], r["dq"], "dq", live)
        self.check(self.dqkv[:, nq * d:(nq + nkv) * d], r["dk"], "dk", live)
        self.check(self.dqkv[:, (nq + nkv) * d:], r["dv"], "dv", live)
        assert bool((self.dqkv.cpu()[dead] == MARK).all())
        return self


# lengths from one token on, around the ends of tiles of 64 and blocks of 128, empty documents, rows of none on both sides
LAYOUTS = {
    "one_token": dict(T=1, lengths=[1]),
    "no_document": dict(T=5, lengths=[]),
    "empty_documents": dict(T=9, lengths=[0, 3, 0, 0, 4, 0], first=1),
    "tokens": dict(T=150, lengths=[1] * 150),
    "tile_ends": dict(T=520, lengths=[64, 63, 65, 1, 127, 129, 64], first=5),
    "block_ends": dict(T=640, lengths=[128, 256, 128], first=128),
    "one_long": dict(T=777, lengths=[777]),
    "ragged": dict(T=1000, lengths=[300, 17, 5, 400, 201], first=0),
    "many_empty": dict(T=200, lengths=[0] * 70 + [100] + [0] * 130 + [90]),
}


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 2, 1, 128), ("bf16", 4, 4, 64), ("f32", 2, 1, 64), ("f32", 2, 2, 24)])
def test_documents(dh, layout, dtype, nq, nkv, d):
    Packed(dh, dtype, nq=nq, nkv=nkv, d=d, **LAYOUTS[layout]).run()


@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 4, 1, 128), ("bf16", 4, 2, 64), ("f32", 3, 1, 128), ("f32", 1, 1, 256), ("f32", 2, 2, 8)])
@pytest.mark.parametrize("cap", [0.0, 5.0, 50.0])
def test_prefixes_and_caps(dh, dtype, nq, nkv, d, cap):
    Packed(dh, dtype, T=460, nq=nq, nkv=nkv, d=d, lengths=[130, 1, 200, 0, 100], prefixes=[130, 1, 70, 0, 9999], first=7, cap=cap, seed=3).run()


@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 8, 1, 128), ("bf16", 32, 8, 64), ("bf16", 3, 3, 128), ("f32", 6, 2, 32)])
def test_head_groups(dh, dtype, nq, nkv, d):
    Packed(dh, dtype, T=333, nq=nq, nkv=nkv, d=d, lengths=[150, 40, 140], prefixes=[20, 0, 64], seed=4).run()


def test_extreme_scores(dh):
    """Scores of thousands: every probability is zero or one, nothing overflows; with a cap they end at the cap."""
    for cap in (0.0, 30.0):
        p = Packed(dh, "bf16", T=300, nq=2, nkv=1, d=128, lengths=[140, 160], cap=cap, seed=5)
        p.qkv[:, :256] *= 64.0
        p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
        p.buffers()
        dh.dh_docs_plan(p.docs)
        p.forward()
        p.backward()
        torch.cuda.synchronize()
        for t in (p.o, p.lse, p.dqkv):
            assert bool(torch.isfinite(t).all())


@pytest.mark.parametrize("dtype,nq,nkv,d", [("bf16", 2, 1, 128), ("bf16", 2, 2, 64), ("f32", 2, 1, 64)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("cap", [0.0, 50.0])
def test_what_is_not_seen_does_not_arrive(dh, dtype, nq, nkv, d, value, cap):
    """A document and the rows of none full of NaNs or infinities, beside others in the same tiles."""
    lengths, first = [50, 30, 100, 20, 150], 3

    def poison(qkv, dout):
        for t in (qkv, dout):
            t[:3] = value
            t[353:] = value
            t[53:83] = value      # the second document
            t[183:203:5] = value  # rows of the fourth

    rows = torch.ones(360, dtype=torch.bool)
    rows[53:83] = rows[183:203] = False
    Packed(dh, dtype, T=360, nq=nq, nkv=nkv, d=d, lengths=lengths, first=first, cap=cap, seed=6).run(poison, rows)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_later_keys_do_not_arrive(dh, dtype, d):
    """Keys and values of the rows behind row 200 of a document are NaNs: the rows before see none of them."""
    p = Packed(dh, dtype, T=300, nq=2, nkv=1, d=d, lengths=[300], seed=7)
    p.qkv[200:, 2 * d:] = float("nan")
    p.qkv_d = p.qkv.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    torch.cuda.synchronize()
    rows = torch.arange(300) < 200
    q = Packed(dh, dtype, T=300, nq=2, nkv=1, d=d, lengths=[300], seed=7)
    p.check(p.o, q.ref()["o"], "o", rows)
    assert bool(torch.isnan(p.o[200:].float()).all())


def test_gradients_against_differences(dh):
    """sum(dout * o) along a direction, float32 inputs: the gradient against a central difference of the float64 formulas."""
    for cap, prefixes in ((0.0, None), (4.0, [10, 33])):
        p = Packed(dh, "f32", T=90, nq=2, nkv=1, d=16, lengths=[40, 45], prefixes=prefixes, first=2, cap=cap, seed=8).run()
        direction = torch.randn(p.qkv.shape, generator=torch.Generator().manual_seed(9)).double()
        direction[~p.live] = 0.0

        def loss(step):
            q = p.qkv.double() + step * direction
            o = R.attention(p.T, 2, 1, 16, cap, p.lo, p.hi, q, p.u)["o"][0]
            return float((o.transpose(0, 1).reshape(p.T, -1) * p.dout.double() * p.live[:, None]).sum())

        h = 1e-4  # the difference's own error: h^2 times a third derivative, and 2^-53 of the loss over h
        want = (loss(h) - loss(-h)) / (2 * h)
        got = float((p.dqkv.cpu().double() * direction * p.live[:, None]).sum())
        size = float((p.dqkv.cpu().double() * direction * p.live[:, None]).abs().sum())
        assert abs(got - want) <= 1e-4 * size


def test_streams_and_replays(dh):
    """Forward and backward captured into a graph together with the table, replayed on other inputs between eager runs: the same bits as eager."""
    p = Packed(dh, "bf16", T=700, nq=4, nkv=1, d=128, lengths=[300, 20, 350], first=4, seed=10)
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step(stream):
        dh.dh_docs_plan(p.docs, stream)
        p.forward(stream)
        p.backward(stream)

    step(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s)
    for k in range(4):
        p.qkv_d.copy_(torch.randn(p.qkv.shape, generator=torch.Generator().manual_seed(20 + k)).to(p.tt))
        p.start.copy_(torch.tensor([k, 10 + 90 * k, 400, 690 - k], dtype=torch.int32))
        torch.cuda.synchronize()
        step(s)
        s.synchronize()
        want = [t.clone() for t in (p.o, p.lse, p.dqkv, p.pos)]
        for t in (p.o, p.lse, p.dqkv, p.delta):
            t.fill_(MARK)
        p.table.fill_(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        live = torch.zeros(p.T, dtype=torch.bool)
        live[k:690 - k] = True
        for a, b in zip((p.o, p.dqkv), (want[0], want[2])):
            assert torch.equal(a[live], b[live]) and bool((a[~live] == MARK).all())
        assert torch.equal(p.lse[:, live], want[1][:, live]) and torch.equal(p.pos, want[3])


def test_starts_out_of_order_touch_nothing_else(dh):
    """Starts that do not ascend or lie outside the rows: whatever rows they give, reads and writes stay in the buffers."""
    for starts in ([5, 3, 40, -7, 200], [1000, 1001, 1002, 2000, 3000], [-50, 20, 10, 500, 90]):
        p = Packed(dh, "bf16", T=100, nq=2, nkv=1, d=64, lengths=[25] * 4, prefixes=[5, 99, -3, 7], seed=11)
        p.start.copy_(torch.tensor(starts, dtype=torch.int32))
        p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
        p.buffers()
        dh.dh_docs_plan(p.docs)
        p.forward()
        p.backward()
        torch.cuda.synchronize()
        pos = p.pos.cpu()
        assert bool(((pos >= 0) & (pos < 100)).all())


@pytest.mark.parametrize("d,cap", [(128, 0.0), (64, 0.0), (128, 50.0), (64, 30.0)])
def test_cut_rows(dh, d, cap):
    """Long documents beside short ones on few heads: blocks of queries and of keys are cut into several units."""
    p = Packed(dh, "bf16", T=2600, nq=2, nkv=1, d=d, lengths=[1900, 30, 600], first=17, cap=cap, seed=12).run()
    cut = p.table[:64].view(torch.int32).cpu()[6::2].tolist()  # blocks that were cut: forward, dQ of heads of 128 and of 64, dK and dV
    assert cut[0] > 0 and cut[2 if d == 64 else 1] > 0 and cut[4 if d == 64 else 3] > 0


def test_cut_rows_beside_what_is_not_finite(dh):
    """Units of a cut row in which keys that the row does not see are NaNs."""
    def poison(qkv, dout):
        qkv[1100:1130] = float("nan")
        dout[1100:1130] = float("inf")

    rows = torch.ones(2000, dtype=torch.bool)
    rows[1100:1130] = False
    Packed(dh, "bf16", T=2000, nq=2, nkv=1, d=128, lengths=[1100, 30, 870], seed=13).run(poison, rows)


def test_two_launches(dh):
    """More blocks of heads than the backward pass takes in one launch."""
    Packed(dh, "bf16", T=1500, nq=96, nkv=32, d=64, lengths=[700, 100, 690], first=5, seed=14).run()


def test_one_prefix_over_everything(dh):
    """Every row sees every key."""
    Packed(dh, "bf16", T=700, nq=2, nkv=1, d=128, lengths=[700], prefixes=[700], seed=15).run()
    Packed(dh, "f32", T=130, nq=2, nkv=1, d=64, lengths=[130], prefixes=[130], seed=15).run()


def test_a_table_for_other_sizes_is_left_alone(dh):
    """Attention whose sizes are not those the table was made for writes nothing."""
    p = Packed(dh, "bf16", T=300, nq=4, nkv=2, d=64, lengths=[300], seed=16)
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.docs.nkv = 1  # the same buffers are large enough
    p.forward()
    torch.cuda.synchronize()
    assert bool((p.o == MARK).all()) and bool((p.lse == MARK).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
@pytest.mark.parametrize("cap", [0.001, 1000.0])
def test_smallest_and_largest_cap(dh, dtype, d, cap):
    Packed(dh, dtype, T=200, nq=2, nkv=1, d=d, lengths=[120, 75], cap=cap, seed=17).run()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 32)])
def test_more_documents_than_the_plan_copies(dh, dtype, d):
    """5000 documents of one token: a row is its own only key, so that o = v exactly, dv = dout and the rest of the gradient is zero."""
    T = 5003
    p = Packed(dh, dtype, T=T, nq=1, nkv=1, d=d, lengths=[1] * 5000, first=2, seed=18)
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    live = slice(2, 5002)
    assert bool((p.pos == 0).all())
    assert torch.equal(p.o.cpu()[live], p.qkv[live, 2 * d:])
    # the score of the backward pass, its p = exp(score - lse), and dout . v - delta are sums of d products in another order than before: d + 8 times 2^-24 of their
    # terms apart (the float32 kernels scale q in one pass and k in the other)
    q, k, v, do = (t[live].double() for t in (p.qkv[:, :d], p.qkv[:, d:2 * d], p.qkv[:, 2 * d:], p.dout))
    apart = (2 * (d + 8) * R.W * (q * k).abs().sum(1) / d ** 0.5)[:, None] + 2 ** -22
    assert bool(((p.dqkv[live, 2 * d:].cpu().double() - do).abs() <= (1.01 * apart + (0 if p.bf16 else R.W)) * do.abs()).all())  # (bf16: p rounds to one)
    off = (2 * (d + 8) * R.W * (do * v).abs().sum(1) / d ** 0.5)[:, None]
    assert bool((p.dqkv[live, :d].cpu().double().abs() <= 1.01 * off * k.abs() + 1e-30).all())
    assert bool((p.dqkv[live, d:2 * d].cpu().double().abs() <= 1.01 * off * q.abs() + 1e-30).all())
    s = (q * k).sum(1) / d ** 0.5
    assert bool(((p.lse[0, live].cpu().double() - s).abs() <= (d + 16) * R.W * ((q * k).abs().sum(1) / d ** 0.5) + 2 ** -22).all())


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 32)])
def test_more_blocks_than_the_plan_weighs(dh, dtype, d):
    """2000 documents of 70 rows: 140000 rows, 1094 blocks."""
    n, docs, T = 70, 2000, 140000
    p = Packed(dh, dtype, T=T, nq=1, nkv=1, d=d, lengths=[n] * docs, seed=19)
    p.qkv_d, p.dout_d = p.qkv.cuda(), p.dout.cuda()
    p.buffers()
    dh.dh_docs_plan(p.docs)
    p.forward()
    p.backward()
    torch.cuda.synchronize()
    q, k, v = (p.qkv_d[:, i * d:(i + 1) * d].double().view(docs, n, d).contiguous() for i in range(3))
    do, sc = p.dout_d.double().view(docs, n, d), d ** -0.5
    hidden = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
    P = torch.softmax((torch.matmul(q, k.transpose(1, 2).contiguous()) * sc).masked_fill(hidden, float("-inf")), 2)
    o = torch.matmul(P, v)
    dS = P * (torch.matmul(do, v.transpose(1, 2).contiguous()) - (do * o).sum(2, keepdim=True)) * sc
    want = torch.cat([torch.matmul(dS, k), torch.matmul(dS.transpose(1, 2).contiguous(), q), torch.matmul(P.transpose(1, 2).contiguous(), do)], 2).view(T, 3 * d)
    # roundings of P, dS, o and the results, half a step each, add up to less than 3 half steps; float32 has its sums of up to 70 + d terms
    tol = 3 * 2.0 ** -8 if p.bf16 else 200 * R.W
    rel = lambda a, b: float((a.double() - b).norm() / b.norm())  # noqa: E731
    assert rel(p.o, o.view(T, d)) <= tol and rel(p.dqkv, want) <= tol
