"""Packed documents, bf16: rows that are made again, next to others of the same block that are not (tests/docs_ref.py holds the formulas and the bounds)."""
import math

import pytest
import torch

from test_gpu_docs_attn import Packed

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [0.0, 50.0])
@pytest.mark.parametrize("which", ["v", "dout"])
def test_waves_beside_one_that_makes_rows_again(dh, d, cap, which):
    """NaNs where the first wave (dK/dV: the first two) of every second block masks them, and the others do not look: the others' rows have the bits they have without NaNs."""
    T = 15 * 128
    i = torch.arange(T)
    first = torch.arange(256, T, 256)
    # v: a document that ends 5 rows before a block, one that reaches 32 rows into it, one behind; dout: one of four rows that ends with a block's first row, one up to its 64th, one behind
    cuts = (first[:, None] + torch.tensor([-5, 32] if which == "v" else [-3, 1, 64])).flatten().tolist()
    lengths = [b - a for a, b in zip([0] + cuts, cuts + [T])]
    clean, p = (Packed(dh, "bf16", T, 2, 2, d, lengths, cap=cap) for _ in range(2))
    a, c = 2 * d, 4 * d
    at = first - 10 if which == "v" else first
    (p.qkv[:, c:] if which == "v" else p.dout)[at] = math.nan
    for x in (clean, p):
        x.qkv_d, x.dout_d = x.qkv.cuda(), x.dout.cuda()
        x.buffers()
        dh.dh_docs_plan(x.docs)
        x.forward()
        x.backward()
    torch.cuda.synchronize()
    seen = (i[None, :] >= p.lo[:, None]) & (i[None, :] < p.hi[:, None])
    grad = seen[:, at].any(1) if which == "v" else torch.isin(i, at)
    hurt = grad if which == "v" else torch.zeros(T, dtype=torch.bool)
    keys = seen[grad].any(0)
    fwd = p.ref()
    p.check(p.o, fwd["o"], "o", ~hurt)
    r = p.ref(dout=p.dout, o_in=p.o.cpu(), lse_in=p.lse.cpu())
    p.check(p.dqkv[:, :a], r["dq"], "dq", ~grad)
    p.check(p.dqkv[:, a:c], r["dk"], "dk", ~keys)
    p.check(p.dqkv[:, c:], r["dv"], "dv", ~keys)
    second = (i // 128 % 2 == 0) & (i >= 256)
    beside, later = second & (i % 128 >= 32), second & (i % 128 >= 64)
    if which == "v":
        beside &= ~hurt  # the next block's NaN lies behind it
        assert int(beside.sum()) == 96 * len(first)
        assert torch.equal(p.o[beside.cuda()], clean.o[beside.cuda()]) and torch.equal(p.lse[:, beside.cuda()], clean.lse[:, beside.cuda()])
    else:
        assert not keys[later].any()
        assert torch.equal(p.dqkv[later.cuda(), a:], clean.dqkv[later.cuda(), a:])
    assert torch.equal(p.dqkv[beside.cuda(), :a], clean.dqkv[beside.cuda(), :a])
