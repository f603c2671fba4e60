"""Dropout that joins the residual stream, through the C ABI: the mask bit for bit, the results against float64."""
import pytest
import torch

import mixers_ref as R

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def test_philox_known_answers():
    """Salmon et al.'s generator: the answers to counters and keys of zeros and of ones, as published with it."""
    assert R.philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert R.philox([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def signed(x):
    return x - 2 ** 64 if x >= 2 ** 63 else x


class Case:
    def __init__(self, dh, tt, T, H, p, bias=True, a=True, key=0x123456789ABCDEF0, step=7, site=3, seed=1):
        self.dh, self.tt, self.T, self.H, self.p, self.site = dh, tt, T, H, p, site
        g = torch.Generator().manual_seed(seed)
        normal = lambda *s: torch.randn(s, generator=g).to(tt)  # noqa: E731
        self.a, self.b, self.bias, self.dout = normal(T, H) if a else None, normal(T, H), normal(H) if bias else None, normal(T, H)
        self.rng = torch.tensor([signed(key), signed(step)], dtype=torch.int64, device="cuda")
        self.dt = dh.DH_BF16 if tt == BF else dh.DH_F32
        self.keep, self.f = R.keep_mask(T, H, p, key, step, site)
        dev = lambda t: None if t is None else t.cuda()  # noqa: E731
        self.a_d, self.b_d, self.bias_d, self.dout_d = dev(self.a), dev(self.b), dev(self.bias), dev(self.dout)
        self.out, self.dx, self.dbias = torch.zeros_like(self.b_d), torch.zeros_like(self.b_d), torch.zeros(H, device="cuda")
        self.wsb = dh.dh_dropout_add_bwd_ws_bytes(T, H)
        self.ws = torch.full((max(16, self.wsb),), 0xff, dtype=torch.uint8, device="cuda")

    def forward(self, stream=None):
        self.dh.dh_dropout_add_fwd(self.dt, self.T, self.H, self.a_d, self.b_d, self.bias_d, self.p, self.rng, self.site, self.out, stream)

    def backward(self, stream=None, accumulate=False, dbias=True):
        self.dh.dh_dropout_add_bwd(self.dt, self.T, self.H, self.dout_d, self.p, self.rng, self.site, self.dx, self.dbias if dbias else None, accumulate, self.ws, self.wsb, stream)

    def check(self, before=None):
        u, keep = R.half_step(self.tt), self.keep.double() * self.f
        x = self.b.double() + (0.0 if self.bias is None else self.bias.double())
        size = self.b.double().abs() + (0.0 if self.bias is None else self.bias.double().abs())
        base = 0.0 if self.a is None else self.a.double()
        val = base + keep * x
        R.check(self.out, (val, 1.01 * u * val.abs() + 4 * R.W * (keep * size + (0.0 if self.a is None else base.abs()))), "out")  # sum, factor, sum, then the result's rounding
        g = keep * self.dout.double()
        R.check(self.dx, (g, 1.01 * u * g.abs() + 2 * R.W * g.abs()), "dx")
        if self.bias is not None:
            total = g.sum(0) + (0.0 if before is None else before.double().cpu())
            R.check(self.dbias, (total, (self.T + 4) * R.W * (g.abs().sum(0) + (0.0 if before is None else before.double().cpu().abs()))), "dbias")


@pytest.mark.parametrize("T,H", [(1, 8), (3, 16), (64, 24), (17, 512), (130, 520), (5, 4096), (1000, 8), (33, 1032)])
@pytest.mark.parametrize("tt", [BF, F])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_both_passes(dh, tt, T, H, p):
    c = Case(dh, tt, T, H, p)
    c.forward()
    c.backward()
    c.check()


@pytest.mark.parametrize("tt", [BF, F])
def test_forms(dh, tt):
    c = Case(dh, tt, 50, 64, 0.3, bias=False)
    c.forward()
    c.backward(dbias=False)
    c.check()
    c = Case(dh, tt, 50, 64, 0.3, a=False, bias=True)
    c.forward()
    c.dbias.fill_(2.0)
    before = c.dbias.clone()
    c.backward(accumulate=True)
    c.check(before)
    c.out = c.b_d  # in place
    c.forward()
    c.dx = c.dout_d
    c.backward(accumulate=False)
    c.check()
    c = Case(dh, tt, 50, 64, 0.3)
    c.out = c.a_d
    c.forward()
    c.backward()
    c.check()


def test_counters(dh):
    """Another key, step or site is another mask, also in the high words; a step's high word does not count."""
    base = Case(dh, F, 40, 256, 0.5)
    base.forward()
    for kw in (dict(key=0x123456789ABCDEF1), dict(key=0xF23456789ABCDEF0), dict(step=8), dict(step=0xFFFFFFFF), dict(site=4), dict(site=0xFFFFFFFF)):
        c = Case(dh, F, 40, 256, 0.5, **kw)
        c.forward()
        c.backward()
        c.check()
        assert 0.3 < float((c.out == base.out).float().mean()) < 0.7
    c = Case(dh, F, 40, 256, 0.5, step=7 + 2 ** 40)
    c.forward()
    assert torch.equal(c.out, base.out)


def test_shares(dh):
    """The share that is kept lies within five standard deviations of 1 - p."""
    T, H = 512, 1024
    x, out = torch.ones((T, H), device="cuda"), torch.empty((T, H), device="cuda")
    rng = torch.tensor([99, 1], dtype=torch.int64, device="cuda")
    for p in (0.01, 0.1, 0.5, 0.9):
        dh.dh_dropout_add_fwd(dh.DH_F32, T, H, None, x, None, p, rng, 0, out)
        kept = float((out != 0).double().mean())
        assert abs(kept - (1 - p)) < 5 * (p * (1 - p) / (T * H)) ** 0.5 + 2.0 ** -17


def test_dropped_infinities(dh):
    c = Case(dh, BF, 20, 64, 0.5)
    c.b_d[~c.keep.cuda()] = float("nan")
    c.dout_d[~c.keep.cuda()] = float("inf")
    c.forward()
    c.backward()
    c.check()


def test_graph_draws_anew_where_the_step_moves(dh):
    c = Case(dh, BF, 300, 256, 0.2)
    graph = torch.cuda.CUDAGraph()
    st = torch.cuda.current_stream()
    with torch.cuda.graph(graph):
        c.forward(torch.cuda.current_stream())
        c.backward(torch.cuda.current_stream())
    for step in (3, 4, 5):
        c.rng[1] = step
        c.keep, c.f = R.keep_mask(c.T, c.H, c.p, 0x123456789ABCDEF0, step, c.site)
        graph.replay()
        st.synchronize()
        c.check()
        graph.replay()
        c.check()


def test_elements_past_32_bits(dh):
    """2^32 elements and a few rows: the last vectors' bits are those of their counters, and the gradient is made likewise."""
    H, T = 8192, 2 ** 19 + 2
    x = torch.ones((T, H), dtype=BF, device="cuda")
    rng = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
    dh.dh_dropout_add_fwd(dh.DH_BF16, T, H, None, x, None, 0.5, rng, 1, x)
    first = (T - 1) * H // 8
    for v in (first, first + 5, T * H // 8 - 1):
        want = [0.0 if b < 32768 else 2.0 for w in R.philox([v & 0xFFFFFFFF, v >> 32, 6, 1], [5, 0]) for b in (w & 0xFFFF, w >> 16)]
        assert x.view(-1)[v * 8:v * 8 + 8].tolist() == want
    n = dh.dh_dropout_add_bwd_ws_bytes(T, H)
    ws, dbias = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(H, device="cuda")
    total = x.sum(0, dtype=torch.float64)
    dh.dh_dropout_add_bwd(dh.DH_BF16, T, H, x, 0.5, rng, 1, x, dbias, False, ws, n)  # keeps what was kept, twice as large
    assert torch.equal(dbias.double(), 2 * total)  # whole numbers below 2^24: exact
