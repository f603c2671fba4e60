"""Window attention, bf16: rows that are made again, next to others of the same block that are not (tests/mixers_ref.py holds the formulas and the bounds)."""
import math

import pytest
import torch

import mixers_ref as R
from test_gpu_window_attn import BF, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", ["v", "dout"])
def test_waves_beside_one_that_makes_rows_again(dh, d, which):
    """NaNs where the first wave (dK/dV: the first two) of every second block masks them, and the others do not look: the others' rows have the bits they have without NaNs."""
    seq, window = 15 * 128, 97
    clean, c = (Case(dh, BF, 1, seq, window, 0, 2, 2, d) for _ in range(2))
    a, b = 2 * d, 4 * d
    i = torch.arange(seq)
    second = (i // 128 % 2 == 0) & (i >= 256)
    if which == "v":
        at = i[second & (i % 128 == 0)] - 97  # in the tile that the first 32 rows of a block share with those before the window
        c.qkv[at, b:] = math.nan
        hurt = c.seen[:, at].any(1)
        keys = c.seen[hurt].any(0)
    else:
        at = i[second & (i % 128 == 0)]       # in the tile of queries that the first 64 keys of a block look at
        c.dout[at] = math.nan
        hurt = torch.zeros(seq, dtype=torch.bool)
        keys = c.seen[at].any(0)
    for x in (clean, c):
        x.upload()
        x.forward()
        x.backward()
    grad = hurt if which == "v" else second & (i % 128 == 0)
    fwd = R.attention(c.seen, 2, 2, d, c.qkv)
    R.check(c.o, fwd["o"], "o", ~hurt[:, None])
    R.check(c.lse, fwd["lse"], "lse", ~hurt[None, :])
    bwd = R.attention(c.seen, 2, 2, d, c.qkv, c.dout, c.o.cpu(), c.lse.cpu())
    R.check(c.dqkv[:, :a], bwd["dq"], "dq", ~grad[:, None])
    R.check(c.dqkv[:, a:b], bwd["dk"], "dk", ~keys[:, None])
    R.check(c.dqkv[:, b:], bwd["dv"], "dv", ~keys[:, None])
    beside = (second & (i % 128 >= 32)).cuda()
    if which == "v":
        assert not hurt[beside.cpu()].any() and int((~hurt & second & (i % 128 < 32)).sum()) == 7 * 32
        assert torch.equal(c.o[beside], clean.o[beside]) and torch.equal(c.lse[:, beside], clean.lse[:, beside])
    else:
        later = (second & (i % 128 >= 64)).cuda()
        assert not keys[later.cpu()].any()
        assert torch.equal(c.dqkv[later, a:], clean.dqkv[later, a:])
        assert torch.equal(c.o, clean.o)
    assert torch.equal(c.dqkv[beside, :a], clean.dqkv[beside, :a])
