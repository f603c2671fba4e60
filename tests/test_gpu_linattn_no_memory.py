"""Linear attention of heads whose decay is minus infinity: each token sees itself alone, so that infinities and NaNs of other tokens and of the state before reach none of its results
(tests/mixers_ref.py holds the formulas and the bounds)."""
import math

import pytest
import torch

import mixers_ref as R
from test_gpu_linattn import BF, F, Case

pytestmark = pytest.mark.gpu
SHAPES = [(BF, 2, 2, 64), (BF, 3, 3, 128), (BF, 8, 2, 128), (BF, 10, 2, 64), (F, 2, 2, 64), (F, 6, 2, 40), (F, 2, 2, 128)]


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def head(n, d, first, count):
    """[1, n * d]: columns of heads [first, first + count)."""
    h = torch.arange(n * d) // d
    return ((h >= first) & (h < first + count))[None, :]


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("tt,nq,nkv,d", SHAPES)
@pytest.mark.parametrize("seq", [1, 45, 64, 330])
def test_each_token_by_itself(dh, tt, nq, nkv, d, seq, bad):
    c = Case(dh, tt, 2, seq, nq, nkv, d, decays=[-math.inf] + [-0.1] * (nkv - 1))
    a, b, g, T = nq * d, (nq + nkv) * d, nq // nkv, 2 * seq
    i = torch.arange(T)
    none = torch.zeros(T, dtype=torch.bool)
    at = {"q": none.clone(), "k": none.clone(), "v": none.clone(), "dout": none.clone()}
    if seq > 1:  # the first sequence's, in one chunk and in others, of the first head alone
        for name, rows in (("q", [3, seq - 2]), ("k", [5, 35, seq - 3]), ("v", [7, 8, 33, seq - 4]), ("dout", [9, 36, seq - 5])):
            at[name][rows] = True
        c.qkv[at["q"], 1] = bad
        c.qkv[at["k"], a + 2] = bad
        c.qkv[at["v"], b + 7] = bad
        c.dout[at["dout"], 4] = bad
    c.state[0, 0, 1::3] = bad
    c.state[1, 0] = bad
    c.dstate[1, 0, :, 5] = bad
    c.upload()
    c.forward()
    c.backward()
    r = c.ref()
    last = i == T - 1  # sees the second sequence's dstate_out

    def check(got, name, n, hurt):
        R.check(got, r[name], name, ~hurt[:, None] | ~head(n, d, 0, g if n == nq else 1))

    check(c.o, "o", nq, at["q"] | at["k"] | at["v"])
    check(c.dqkv[:, :a], "dq", nq, at["k"] | at["v"] | at["dout"])
    check(c.dqkv[:, a:b], "dk", nkv, at["v"] | at["q"] | at["dout"] | last)
    check(c.dqkv[:, b:], "dv", nkv, at["k"] | at["q"] | at["dout"] | last)
    R.check(c.state_out, r["state"], "state")
    R.check(c.dstate_in, r["dstate"], "dstate")
    assert (c.dstate_in[:, 0] == 0).all()
    for name, t in (("q", c.o), ("k", c.o), ("v", c.o), ("dout", c.dqkv[:, :a])):
        if seq > 1:
            assert not torch.isfinite(t[at[name].cuda(), :d].float()).all(1).any(), name
    c.forward(state_out=False)
    c.backward(dstate_in=False)
    check(c.o, "o", nq, at["q"] | at["k"] | at["v"])
    check(c.dqkv[:, a:b], "dk", nkv, at["v"] | at["q"] | at["dout"] | last)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("tt,nq,nkv,d", SHAPES + [(BF, 20, 2, 128)])
def test_single_tokens(dh, tt, nq, nkv, d, bad):
    c = Case(dh, tt, 3, 1, nq, nkv, d, decays=[-math.inf] + [-0.1] * (nkv - 1))
    c.state[:2, 0] = bad
    c.upload()
    out = torch.full_like(c.state_d, 3.0)
    dh.dh_linattn_step(c.dt, 3, nq, nkv, d, c.scale, c.decay_d, torch.tensor([5, 1, 7], dtype=torch.int32, device="cuda"), c.qkv_d, c.state_d, out, c.o)
    r = c.ref()
    R.check(c.o, r["o"], "o")
    R.check(out, r["state"], "state")
    dh.dh_linattn_step(c.dt, 3, nq, nkv, d, c.scale, c.decay_d, None, c.qkv_d, c.state_d, c.state_d, c.o)
    R.check(c.o, r["o"], "o")
    R.check(c.state_d, r["state"], "state")
