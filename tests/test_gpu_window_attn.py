"""Attention with a sliding window and sinks through the C ABI, against float64 (tests/mixers_ref.py holds the formulas and the bounds)."""
import math

import pytest
import torch

import mixers_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
MARK = 7.0


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


class Case:
    def __init__(self, dh, tt, batch, seq, window, sinks, nq, nkv, d, seed=1):
        self.dh, self.tt, self.batch, self.seq, self.window, self.sinks, self.nq, self.nkv, self.d = dh, tt, batch, seq, window, sinks, nq, nkv, d
        self.T = T = batch * seq
        self.args = (dh.DH_BF16 if tt == BF else dh.DH_F32, batch, seq, window, sinks, nq, nkv, d)
        g = torch.Generator().manual_seed(seed)
        self.qkv = torch.randn((T, (nq + 2 * nkv) * d), generator=g)
        self.qkv[:, :nq * d] *= 2.0
        self.qkv, self.dout = self.qkv.to(tt), torch.randn((T, nq * d), generator=g).to(tt)
        self.seen = R.seen_by(batch, seq, window, sinks)

    def upload(self):
        full = lambda *shape, t=self.tt: torch.full(shape, MARK, dtype=t, device="cuda")  # noqa: E731
        self.qkv_d, self.dout_d = self.qkv.cuda(), self.dout.cuda()
        self.o, self.lse, self.dqkv, self.delta = full(self.T, self.nq * self.d), full(self.nq, self.T, t=F), full(*self.qkv.shape), full(self.nq, self.T, t=F)
        self.wsb = max(self.dh.dh_attn_window_fwd_workspace_bytes(*self.args), self.dh.dh_attn_window_bwd_workspace_bytes(*self.args))
        self.ws = torch.full((max(16, self.wsb),), 0xff, dtype=torch.uint8, device="cuda")  # NaNs
        return self

    def forward(self, stream=None):
        self.dh.dh_attn_window_fwd(*self.args, self.qkv_d, self.o, self.lse, self.ws, self.wsb, stream)

    def backward(self, stream=None):
        self.dh.dh_attn_window_bwd(*self.args, self.qkv_d, self.o, self.dout_d, self.lse, self.dqkv, self.delta, self.ws, self.wsb, stream)

    def results(self):
        return [t.clone() for t in (self.o, self.lse, self.dqkv, self.delta)]

    def check(self, rows=None, keys=None):
        """rows, keys: which rows' results, and which keys' gradients, count."""
        fwd = R.attention(self.seen, self.nq, self.nkv, self.d, self.qkv)
        r = None if rows is None else rows[:, None]
        R.check(self.o, fwd["o"], "o", r)
        R.check(self.lse, fwd["lse"], "lse", None if rows is None else rows[None, :])
        bwd = R.attention(self.seen, self.nq, self.nkv, self.d, self.qkv, self.dout, self.o.cpu(), self.lse.cpu())
        a, b = self.nq * self.d, (self.nq + self.nkv) * self.d
        c = None if keys is None else keys[:, None]
        R.check(self.dqkv[:, :a], bwd["dq"], "dq", r)
        R.check(self.dqkv[:, a:b], bwd["dk"], "dk", c)
        R.check(self.dqkv[:, b:], bwd["dv"], "dv", c)


SHAPES = [(1, 1, 1, 0), (2, 1, 5, 3), (1, 63, 1, 0), (1, 64, 16, 1), (3, 65, 64, 4), (1, 130, 33, 40), (2, 200, 64, 0), (1, 257, 100, 70), (1, 300, 1000, 2), (1, 300, 7, 400),
          (1, 513, 128, 64), (2, 333, 2, 130), (1, 700, 2 ** 31 - 1, 2 ** 31 - 1), (1, 640, 256, 16), (1, 1000, 190, 33)]


@pytest.mark.parametrize("batch,seq,window,sinks", SHAPES)
@pytest.mark.parametrize("tt,nq,nkv,d", [(BF, 2, 2, 64), (BF, 4, 1, 128), (BF, 6, 2, 64), (F, 2, 2, 64), (F, 3, 1, 40)])
def test_both_passes(dh, tt, nq, nkv, d, batch, seq, window, sinks):
    c = Case(dh, tt, batch, seq, window, sinks, nq, nkv, d, seed=seq + window).upload()
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("tt,nq,nkv,d", [(F, 1, 1, 8), (F, 2, 1, 128), (F, 5, 5, 24), (BF, 16, 1, 64), (BF, 8, 8, 128), (BF, 12, 4, 128)])
def test_head_layouts(dh, tt, nq, nkv, d):
    c = Case(dh, tt, 2, 150, 50, 5, nq, nkv, d).upload()
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("tt,d", [(BF, 64), (BF, 128), (F, 64)])
def test_a_whole_window_is_causal_attention(dh, tt, d):
    batch, seq, nq, nkv = 2, 391, 4, 2
    c = Case(dh, tt, batch, seq, seq, 0, nq, nkv, d).upload()
    c.forward()
    a = (c.args[0], batch, seq, nq, nkv, d)
    o, lse, dqkv, delta = torch.zeros_like(c.o), torch.zeros_like(c.lse), torch.zeros_like(c.dqkv), torch.zeros_like(c.delta)
    n = max(16, dh.dh_attn_fwd_workspace_bytes(*a), dh.dh_attn_bwd_workspace_bytes(*a))
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    dh.dh_attn_fwd(*a, c.qkv_d, o, lse, ws, n)
    fwd = R.attention(c.seen, nq, nkv, d, c.qkv)
    R.check(c.o, (o.double().cpu(), 2 * fwd["o"][1]), "o")  # either side lies within the bound of the same number
    R.check(c.lse, (lse.double().cpu(), 2 * fwd["lse"][1]), "lse")
    c.o, c.lse = o, lse
    c.backward()
    dh.dh_attn_bwd(*a, c.qkv_d, o, c.dout_d, lse, dqkv, delta, ws, n)
    bwd = R.attention(c.seen, nq, nkv, d, c.qkv, c.dout, o.cpu(), lse.cpu())
    R.check(c.dqkv, (dqkv.double().cpu(), 2 * torch.cat([bwd[k][1] for k in ("dq", "dk", "dv")], 1)), "dqkv")


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("tt,nq,nkv,d,seq,window,sinks", [(BF, 4, 2, 128, 420, 70, 6), (BF, 2, 2, 64, 420, 70, 6), (F, 2, 1, 64, 420, 70, 6),
                                                          (BF, 2, 1, 128, 1500, 1300, 70),  # parts of a walk over keys
                                                          (BF, 40, 8, 128, 1300, 200, 4),   # as many blocks as take two launches
                                                          (BF, 4, 4, 64, 700, 400, 130)])
def test_what_a_row_does_not_see_does_not_reach_it(dh, tt, nq, nkv, d, seq, window, sinks, bad):
    at, last = [3, 100, 101, 260, seq - 1], seq - 1
    c = Case(dh, tt, 1, seq, window, sinks, nq, nkv, d)
    a, b = nq * d, (nq + nkv) * d
    c.qkv[100, b:] = bad                     # a value
    c.qkv[101, a + 3] = bad                  # a key's element
    c.qkv[260, b + 5] = bad
    c.qkv[last, :a] = bad                    # the last row's query: it sees the sinks
    c.qkv[3, b + 1::7] = bad                 # a sink, which every later row sees
    if d == 64:
        c.qkv[3, b + 1::7] = 0.5
        at.remove(3)
    c.dout[300, 2] = bad
    c.upload()
    c.forward()
    c.backward()
    hurt = c.seen[:, at].any(1) | torch.tensor([i == last for i in range(seq)])       # rows with such a key or query
    grad = hurt | torch.tensor([i == 300 for i in range(seq)])
    keys = c.seen[grad].any(0)                                                       # keys that a hurt row sees
    fwd = R.attention(c.seen, nq, nkv, d, c.qkv)
    R.check(c.o, fwd["o"], "o", ~hurt[:, None])
    R.check(c.lse, fwd["lse"], "lse", ~hurt[None, :])
    bwd = R.attention(c.seen, nq, nkv, d, c.qkv, c.dout, c.o.cpu(), c.lse.cpu())
    R.check(c.dqkv[:, :a], bwd["dq"], "dq", ~grad[:, None])
    R.check(c.dqkv[:, a:b], bwd["dk"], "dk", ~keys[:, None])
    R.check(c.dqkv[:, b:], bwd["dv"], "dv", ~keys[:, None])
    assert not torch.isfinite(c.o[100].float()).all() and not torch.isfinite(c.dqkv[300].float()).all()


@pytest.mark.parametrize("nq,nkv,d,seq,window,sinks", [(4, 2, 128, 420, 70, 6), (2, 2, 64, 420, 70, 0), (2, 1, 128, 1500, 1300, 70), (40, 8, 128, 1300, 200, 4)])
@pytest.mark.parametrize("which", ["qkv", "dout"])
def test_nothing_but_nans_from_a_row_on(dh, nq, nkv, d, seq, window, sinks, which):
    """A step that has diverged: what sees such a row is a NaN, what sees none is as without them."""
    c, first = Case(dh, BF, 1, seq, window, sinks, nq, nkv, d), seq // 2
    (c.qkv if which == "qkv" else c.dout)[first:] = math.nan
    c.upload()
    c.forward()
    c.backward()
    a = nq * d
    if which == "qkv":
        assert torch.isnan(c.o[first:].float()).all() and torch.isnan(c.lse[:, first:]).all()
    assert torch.isnan(c.dqkv[first:].float()).all()
    fine, keys = torch.arange(seq) < first, ~c.seen[first:].any(0)
    fwd = R.attention(c.seen, nq, nkv, d, c.qkv)
    R.check(c.o, fwd["o"], "o", fine[:, None])
    bwd = R.attention(c.seen, nq, nkv, d, c.qkv, c.dout, c.o.cpu(), c.lse.cpu())
    R.check(c.dqkv[:, :a], bwd["dq"], "dq", fine[:, None])
    b = a + nkv * d
    R.check(c.dqkv[:, a:b], bwd["dk"], "dk", keys[:, None])
    R.check(c.dqkv[:, b:], bwd["dv"], "dv", keys[:, None])
    assert torch.isnan(c.dqkv[~keys.cuda(), a:].float()).all()


def test_scores_of_minus_infinity(dh):
    """Keys of minus infinity weigh nothing beside others, and a row with nothing else has lse minus infinity."""
    for tt, d in ((BF, 64), (BF, 128), (F, 64)):
        c = Case(dh, tt, 1, 90, 8, 2, 1, 1, d)
        c.qkv[:, :d] = 1.0
        c.qkv[0:2, d:2 * d] = -math.inf
        c.qkv[50, d:2 * d] = -math.inf
        c.upload()
        c.forward()
        assert torch.isneginf(c.lse[0, :2]).all() and torch.isnan(c.o[:2].float()).all(), (tt, d)
        keep = c.qkv.clone()
        fwd = R.attention(c.seen, 1, 1, d, keep)
        x = torch.arange(90)
        R.check(c.o, (fwd["o"][0], torch.full_like(fwd["o"][0], 0.05)), "o", ((x > 1) & (x != 50))[:, None])
        R.check(c.lse, (fwd["lse"][0], torch.full_like(fwd["lse"][0], 0.05)), "lse", ((x > 1) & (x != 50))[None, :])


@pytest.mark.parametrize("tt,d", [(BF, 64), (BF, 128), (F, 64)])
def test_bits_streams_and_graphs(dh, tt, d):
    """The same bits on every call, on another stream, and in replays of a captured graph between eager calls."""
    c = Case(dh, tt, 2, 530, 100, 9, 8, 2, d).upload()
    other = Case(dh, tt, 2, 530, 100, 9, 8, 2, d, seed=5).upload()
    c.forward()
    c.backward()
    first = c.results()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    c.upload()
    torch.cuda.synchronize()
    c.forward(st)
    c.backward(st)
    st.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, c.results()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(torch.cuda.current_stream())
        c.backward(torch.cuda.current_stream())
    for _ in range(3):
        for t in (c.o, c.lse, c.dqkv, c.delta):
            t.fill_(3.0)
        other.forward()
        other.backward()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, c.results()))


def test_gradients_against_differences(dh):
    c = Case(dh, F, 1, 40, 9, 3, 2, 1, 16).upload()
    c.forward()
    c.backward()
    g = torch.Generator().manual_seed(4)
    for _ in range(3):
        step = torch.randn(c.qkv.shape, generator=g, dtype=torch.float64)
        sides = []
        for s in (1e-4, -1e-4):
            x = c.qkv.double() + s * step
            q, k, v = (R.heads(t, n, 16).repeat_interleave(2 // n, 0) for t, n in ((x[:, :32], 2), (x[:, 32:48], 1), (x[:, 48:], 1)))
            y = (torch.matmul(q, k.transpose(1, 2)) / 4.0).masked_fill(~c.seen, -math.inf)
            sides.append(float((R.rows(torch.matmul(torch.softmax(y, 2), v)) * c.dout.double()).sum()))
        want = (sides[0] - sides[1]) / 2e-4
        got = float((c.dqkv.double().cpu() * step).sum())
        assert abs(got - want) <= 1e-4 * float((c.dqkv.double().cpu() * step).abs().sum())  # float32 results of O(1) sums; the difference itself is good to 1e-8


# ------------------------------------------------------------------------------------ single tokens
def step_case(dh, tt, positions, rows, window, sinks, nq, nkv, d, seed=2):
    B = len(positions)
    g = torch.Generator().manual_seed(seed)
    history = [torch.randn((max(p, 0), 2 * nkv * d), generator=g).to(tt) for p in positions]
    qkv = torch.randn((B, (nq + 2 * nkv) * d), generator=g)
    qkv[:, :nq * d] *= 2.0
    qkv = qkv.to(tt)
    kv = torch.full((B, rows, 2 * nkv * d), math.nan, dtype=tt)  # rows that no position has been put into
    row = lambda p: p if p < rows else sinks + (p - sinks) % (rows - sinks)  # noqa: E731
    for b, h in enumerate(history):
        for p in range(len(h)):
            kv[b, row(p)] = h[p]
    kv_d, o = kv.cuda(), torch.full((B, nq * d), MARK, dtype=tt, device="cuda")
    a = (dh.DH_BF16 if tt == BF else dh.DH_F32, B, rows, window, sinks, nq, nkv, d)
    n = dh.dh_attn_window_step_workspace_bytes(*a)
    ws = torch.full((max(16, n),), 0xff, dtype=torch.uint8, device="cuda")
    pos = torch.tensor(positions, dtype=torch.int32, device="cuda")
    dh.dh_attn_window_step(*a, pos, qkv.cuda(), kv_d, o, ws, n)
    for b, p in enumerate(positions):
        if p < 0:
            assert (o[b] == MARK).all() and torch.equal(kv_d[b].cpu().view(torch.uint8), kv[b].view(torch.uint8))
            continue
        kv[b, row(p)] = qkv[b, nq * d:]
        assert torch.equal(kv_d[b].cpu().view(torch.uint8), kv[b].view(torch.uint8)), (b, p)
        seen = [j for j in range(p + 1) if j > p - window or j < sinks]
        every = torch.cat([history[b], qkv[b:b + 1, nq * d:]])[seen]
        whole = torch.cat([torch.zeros((len(seen), nq * d), dtype=tt), every], 1)
        whole[-1, :nq * d] = qkv[b, :nq * d]
        mask = torch.zeros((len(seen), len(seen)), dtype=torch.bool)
        mask[-1] = True
        mask[:, 0] = True
        val, err = R.attention(mask, nq, nkv, d, whole)["o"]
        R.check(o[b], (val[-1], err[-1]), "o of sequence %d at %d" % (b, p))


@pytest.mark.parametrize("tt,nq,nkv,d", [(BF, 4, 1, 128), (BF, 8, 8, 64), (BF, 12, 1, 128), (BF, 3, 1, 64), (F, 4, 2, 64), (F, 1, 1, 40), (F, 20, 2, 128), (F, 2, 2, 8)])
@pytest.mark.parametrize("rows,window,sinks", [(20, 16, 4), (64, 33, 0), (300, 150, 70), (1, 1, 0), (900, 700, 3)])
def test_single_tokens(dh, tt, nq, nkv, d, rows, window, sinks):
    step_case(dh, tt, [0, -1, 1, rows - 1, rows, rows + 1, 3 * rows + 5, window, sinks], rows, window, sinks, nq, nkv, d)


def test_single_tokens_of_one_long_sequence(dh):
    step_case(dh, BF, [9999], 5000, 4900, 100, 8, 1, 128)
    step_case(dh, BF, [4000], 5000, 4900, 100, 8, 8, 64)


def test_steps_follow_the_forward_pass(dh):
    """Token by token through a bounded cache gives the rows of the whole forward pass."""
    seq, window, sinks, nq, nkv, d, rows = 60, 12, 3, 4, 2, 64, 20
    c = Case(dh, F, 1, seq, window, sinks, nq, nkv, d).upload()
    c.forward()
    kv, o = torch.full((1, rows, 2 * nkv * d), math.nan, device="cuda"), torch.zeros((1, nq * d), device="cuda")
    n = dh.dh_attn_window_step_workspace_bytes(dh.DH_F32, 1, rows, window, sinks, nq, nkv, d)
    ws = torch.zeros(max(16, n), dtype=torch.uint8, device="cuda")
    for t in range(seq):
        dh.dh_attn_window_step(dh.DH_F32, 1, rows, window, sinks, nq, nkv, d, torch.tensor([t], dtype=torch.int32, device="cuda"), c.qkv_d[t:t + 1], kv, o, ws, n)
        assert torch.allclose(o[0], c.o[t], rtol=1e-5, atol=1e-5), t


def test_cache_offsets_past_32_bits(dh):
    """5 GB of cache: the last sequence's rows lie behind 2^31 elements."""
    B, rows, window, sinks, nkv, d = 41, 16384, 64, 2, 16, 128
    kv = torch.zeros((B, rows, 2 * nkv * d), dtype=BF, device="cuda")
    assert kv.numel() > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(1)
    kv[B - 1, -200:] = torch.randn((200, 2 * nkv * d), generator=g, device="cuda").to(BF)
    qkv = torch.randn((B, 3 * nkv * d), generator=g, device="cuda").to(BF)
    pos = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    pos[B - 1] = rows - 1
    o = torch.zeros((B, nkv * d), dtype=BF, device="cuda")
    a = (dh.DH_BF16, B, rows, window, sinks, nkv, nkv, d)
    n = dh.dh_attn_window_step_workspace_bytes(*a)
    ws = torch.zeros(max(16, n), dtype=torch.uint8, device="cuda")
    dh.dh_attn_window_step(*a, pos, qkv, kv, o, ws, n)
    seen = torch.cat([kv[B - 1, :sinks], kv[B - 1, rows - window:]]).cpu()
    assert torch.equal(seen[-1], qkv[B - 1, nkv * d:].cpu())
    whole = torch.cat([torch.zeros((len(seen), nkv * d), dtype=BF), seen], 1)
    whole[-1, :nkv * d] = qkv[B - 1, :nkv * d].cpu()
    mask = torch.zeros((len(seen), len(seen)), dtype=torch.bool)
    mask[-1], mask[:, 0] = True, True
    val, err = R.attention(mask, nkv, nkv, d, whole)["o"]
    R.check(o[B - 1], (val[-1], err[-1]), "o")
    assert (o[:B - 1] == 0).all()
