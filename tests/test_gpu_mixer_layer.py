"""Window attention, linear attention and dropout as a model uses them: two half layers in training, one with each mixer, whose results join the residual stream through dropout; and the same
model token by token."""
import math

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


class Model:
    """x1 = x + drop(window(rope(x Wa)) Wb + ba);  y = x1 + drop(linear(x1 Wc) Wd + bd)."""
    BATCH, SEQ, H, NQ, NKV, D, WINDOW, SINKS, P, SITES = 2, 150, 128, 4, 2, 64, 40, 3, 0.2, (11, 12)

    def __init__(self, dh, tt, seq=None):
        self.dh, self.tt, self.seq = dh, tt, seq or self.SEQ
        self.t = dh.DH_BF16 if tt == BF else dh.DH_F32
        g = torch.Generator().manual_seed(3)
        H, D, w = self.H, self.D, (self.NQ + 2 * self.NKV) * self.D
        self.T = self.BATCH * self.seq
        normal = lambda s, std: (torch.randn(s, generator=g) * std).to(tt)  # noqa: E731
        self.W = {"a": normal((H, w), H ** -0.5), "b": normal((self.NQ * D, H), (self.NQ * D) ** -0.5), "c": normal((H, w), H ** -0.5), "d": normal((self.NQ * D, H), (self.NQ * D) ** -0.5)}
        self.bias = [normal((H,), 0.1), normal((H,), 0.1)]
        self.x, self.dy = normal((self.BATCH, self.SEQ, H), 1.0)[:, :self.seq].reshape(-1, H).contiguous(), normal((self.BATCH, self.SEQ, H), 1.0)[:, :self.seq].reshape(-1, H).contiguous()
        self.log_decay = torch.tensor([-0.2, -0.01])
        self.rng = torch.tensor([1234567, 5], dtype=torch.int64, device="cuda")
        self.Wd, self.biasd = {k: v.cuda() for k, v in self.W.items()}, [b.cuda() for b in self.bias]
        self.xd, self.dyd, self.decay = self.x.cuda(), self.dy.cuda(), self.log_decay.cuda()
        z = lambda *s, t=tt: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
        T = self.T
        self.qkv, self.o, self.proj = [z(T, w), z(T, w)], [z(T, self.NQ * D), z(T, self.NQ * D)], z(T, H)
        self.lse, self.delta, self.x1, self.y = z(self.NQ, T, t=F), z(self.NQ, T, t=F), z(T, H), z(T, H)
        self.g = {k: z(*v.shape, t=F) for k, v in self.W.items()}
        self.gbias = [z(H, t=F), z(H, t=F)]
        self.dproj, self.do, self.dqkv, self.dmix, self.dx1, self.dx = z(T, H), z(T, self.NQ * D), z(T, w), z(T, H), z(T, H), z(T, H)
        self.wa = (self.t, self.BATCH, self.seq, self.WINDOW, self.SINKS, self.NQ, self.NKV, D)
        self.la = (self.t, self.BATCH, self.seq, self.NQ, self.NKV, D)
        n = max(dh.dh_attn_window_fwd_workspace_bytes(*self.wa), dh.dh_attn_window_bwd_workspace_bytes(*self.wa), dh.dh_linattn_fwd_workspace_bytes(*self.la),
                dh.dh_linattn_bwd_workspace_bytes(*self.la), dh.dh_dropout_add_bwd_ws_bytes(T, H))
        self.wsb, self.ws = n, torch.full((max(16, n),), 0xff, dtype=torch.uint8, device="cuda")  # one workspace, call after call
        self.scale = 1.0 / math.sqrt(D)

    def mm(self, a, b, out, ta=False, tb=False, acc=False):
        M, K = (a.shape[1], a.shape[0]) if ta else a.shape
        self.dh.dh_gemm(self.t, ta, tb, M, b.shape[0] if tb else b.shape[1], K, a, b, out, acc, None, 0, torch.cuda.current_stream())

    def forward(self):
        dh, st = self.dh, torch.cuda.current_stream()
        w = (self.NQ + 2 * self.NKV) * self.D
        self.mm(self.xd, self.Wd["a"], self.qkv[0])
        dh.dh_rope(self.t, self.T, self.seq, self.NQ + self.NKV, self.D, w, 1e4, False, self.qkv[0], st)
        dh.dh_attn_window_fwd(*self.wa, self.qkv[0], self.o[0], self.lse, self.ws, self.wsb, st)
        self.mm(self.o[0], self.Wd["b"], self.proj)
        dh.dh_dropout_add_fwd(self.t, self.T, self.H, self.xd, self.proj, self.biasd[0], self.P, self.rng, self.SITES[0], self.x1, st)
        self.mm(self.x1, self.Wd["c"], self.qkv[1])
        dh.dh_linattn_fwd(*self.la, self.scale, self.decay, self.qkv[1], None, self.o[1], None, self.ws, self.wsb, st)
        self.mm(self.o[1], self.Wd["d"], self.proj)
        dh.dh_dropout_add_fwd(self.t, self.T, self.H, self.x1, self.proj, self.biasd[1], self.P, self.rng, self.SITES[1], self.y, st)

    def backward(self):
        dh, st = self.dh, torch.cuda.current_stream()
        w = (self.NQ + 2 * self.NKV) * self.D
        for t in (*self.g.values(), *self.gbias):
            t.zero_()
        dh.dh_dropout_add_bwd(self.t, self.T, self.H, self.dyd, self.P, self.rng, self.SITES[1], self.dproj, self.gbias[1], True, self.ws, self.wsb, st)
        self.mm(self.o[1], self.dproj, self.g["d"], ta=True, acc=True)
        self.mm(self.dproj, self.Wd["d"], self.do, tb=True)
        dh.dh_linattn_bwd(*self.la, self.scale, self.decay, self.qkv[1], None, self.do, None, self.dqkv, None, self.ws, self.wsb, st)
        self.mm(self.x1, self.dqkv, self.g["c"], ta=True, acc=True)
        self.mm(self.dqkv, self.Wd["c"], self.dmix, tb=True)
        dh.dh_add(self.t, self.T * self.H, self.dmix, self.dyd, self.dx1, st)
        dh.dh_dropout_add_bwd(self.t, self.T, self.H, self.dx1, self.P, self.rng, self.SITES[0], self.dproj, self.gbias[0], True, self.ws, self.wsb, st)
        self.mm(self.o[0], self.dproj, self.g["b"], ta=True, acc=True)
        self.mm(self.dproj, self.Wd["b"], self.do, tb=True)
        dh.dh_attn_window_bwd(*self.wa, self.qkv[0], self.o[0], self.do, self.lse, self.dqkv, self.delta, self.ws, self.wsb, st)
        dh.dh_rope(self.t, self.T, self.seq, self.NQ + self.NKV, self.D, w, 1e4, True, self.dqkv, st)
        self.mm(self.xd, self.dqkv, self.g["a"], ta=True, acc=True)
        self.mm(self.dqkv, self.Wd["a"], self.dmix, tb=True)
        dh.dh_add(self.t, self.T * self.H, self.dmix, self.dx1, self.dx, st)

    def results(self):
        return {"y": self.y, "dx": self.dx, **{"W" + k: v for k, v in self.g.items()}, "ba": self.gbias[0], "bd": self.gbias[1]}


def reference(m):
    """The same in float64 by automatic differentiation."""
    B, n, H, NQ, NKV, D = m.BATCH, m.seq, m.H, m.NQ, m.NKV, m.D
    leaf = lambda t: t.double().requires_grad_()  # noqa: E731
    x, W, bias = leaf(m.x), {k: leaf(v) for k, v in m.W.items()}, [leaf(b) for b in m.bias]

    def split(qkv):
        t = qkv.view(B, n, NQ + 2 * NKV, D).transpose(1, 2)
        return t[:, :NQ], t[:, NQ:NQ + NKV].repeat_interleave(NQ // NKV, 1), t[:, NQ + NKV:].repeat_interleave(NQ // NKV, 1)

    def join(o):
        return o.transpose(1, 2).reshape(B * n, NQ * D)

    def rope(t):
        a = torch.arange(n, dtype=torch.float64)[:, None] * 1e4 ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
        u, v = t[..., :D // 2], t[..., D // 2:]
        return torch.cat([u * a.cos() - v * a.sin(), v * a.cos() + u * a.sin()], -1)

    def drop(t, site):
        keep, f = R.keep_mask(B * n, H, m.P, 1234567, 5, site)
        return t * keep.double() * f

    q, k, v = split(x @ W["a"])
    i = torch.arange(n)
    seen = (i[None, :] <= i[:, None]) & ((i[None, :] > i[:, None] - m.WINDOW) | (i[None, :] < m.SINKS))
    y = (rope(q) @ rope(k).transpose(2, 3) * m.scale).masked_fill(~seen, -math.inf)
    x1 = x + drop(join(torch.softmax(y, 3) @ v) @ W["b"] + bias[0], m.SITES[0])
    q, k, v = split(x1 @ W["c"])
    apart = (i[:, None] - i[None, :]).clamp(min=0).double()
    weight = torch.exp(m.log_decay.double().repeat_interleave(NQ // NKV)[:, None, None] * apart) * (i[None, :] <= i[:, None])
    out = x1 + drop(join((q @ k.transpose(2, 3) * weight * m.scale) @ v) @ W["d"] + bias[1], m.SITES[1])
    out.backward(m.dy.double())
    return {"y": out.detach(), "dx": x.grad, **{"W" + k: v.grad for k, v in W.items()}, "ba": bias[0].grad, "bd": bias[1].grad}


@pytest.mark.parametrize("tt", [F, BF])
def test_training_step(dh, tt):
    """Ten operators in a row, each of which rounds its results (half a step of the type, and of bf16's probabilities, scores and states once more) and adds up at most 600 float32 terms:
    relative norms below 30 roundings of the type and ten sums."""
    m = Model(dh, tt)
    m.forward()
    m.backward()
    want, bound = reference(m), 30 * R.half_step(tt) + 10 * 600 * R.W
    for name, got in m.results().items():
        off = float((got.double().cpu() - want[name]).norm() / want[name].norm())
        assert off <= bound, (name, off, bound)


@pytest.mark.parametrize("tt", [F, BF])
def test_step_in_a_graph(dh, tt):
    """The whole step captured and replayed, also beside eager work on other data, gives the eager bits."""
    m, other = Model(dh, tt), Model(dh, tt)
    m.forward()
    m.backward()
    first = {k: v.clone() for k, v in m.results().items()}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        m.forward()
        m.backward()
    for _ in range(3):
        for t in m.results().values():
            t.fill_(9.0)
        other.xd.normal_()
        other.forward()
        other.backward()
        graph.replay()
        torch.cuda.synchronize()
        for k, v in m.results().items():
            assert torch.equal(v, first[k]), k


def test_token_by_token(dh):
    """Without dropout, the rows of the forward pass one at a time: a bounded cache and a state a sequence."""
    m = Model(dh, F, seq=70)
    m.P = 0.0
    m.forward()
    B, H, NQ, NKV, D, rows = m.BATCH, m.H, m.NQ, m.NKV, m.D, m.WINDOW + m.SINKS
    w = (NQ + 2 * NKV) * D
    kv, state = torch.full((B, rows, 2 * NKV * D), math.nan, device="cuda"), torch.full((B, NKV, D, D), math.nan, device="cuda")
    a = (dh.DH_F32, B, rows, m.WINDOW, m.SINKS, NQ, NKV, D)
    n = dh.dh_attn_window_step_workspace_bytes(*a)
    ws = torch.zeros(max(16, n), dtype=torch.uint8, device="cuda")
    qkv, o, proj, x1, y = (torch.zeros(s, device="cuda") for s in ((B, w), (B, NQ * D), (B, H), (B, H), (B, H)))
    for t in range(m.seq):
        x, pos = m.xd.view(B, m.seq, H)[:, t].contiguous(), torch.full((B,), t, dtype=torch.int32, device="cuda")
        m.mm(x, m.Wd["a"], qkv)
        dh.dh_rope_at(dh.DH_F32, B, 1, t, NQ + NKV, D, w, 1e4, False, qkv)
        dh.dh_attn_window_step(*a, pos, qkv, kv, o, ws, n)
        m.mm(o, m.Wd["b"], proj)
        dh.dh_dropout_add_fwd(dh.DH_F32, B, H, x, proj, m.biasd[0], 0.0, m.rng, 0, x1)
        m.mm(x1, m.Wd["c"], qkv)
        dh.dh_linattn_step(dh.DH_F32, B, NQ, NKV, D, m.scale, m.decay, pos, qkv, state, state, o)
        m.mm(o, m.Wd["d"], proj)
        dh.dh_dropout_add_fwd(dh.DH_F32, B, H, x1, proj, m.biasd[1], 0.0, m.rng, 0, y)
        want = m.y.view(B, m.seq, H)[:, t]
        assert float((y - want).norm() / want.norm()) <= 30 * R.W + 10 * 600 * R.W, t  # as a training step's
