"""Starts of documents that do not ascend or lie outside the rows: what the table may hold then, and that nothing outside the buffers is written.  (Which row goes to which
document is not specified.)"""
import pytest
import torch

pytestmark = pytest.mark.gpu
BYTE, PAD = 0xa5, 4096  # what lies around every buffer, and how many bytes of it on each side


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


# [100, 0, 100, 99, 98]: every row lies before the first start, and yet between the second and the third
SMALL = [[5, 3, 40, -7, 200], [1000, 1001, 1002, 2000, 3000], [-50, 20, 10, 500, 90], [200, 0, 300, 300, 1], [100, 0, 100, 99, 98], [60, 0, 70, 10, 30], [0, 100, 0, 100, 0]]
LARGE = [[17, 2400, 60, 1900, 2600], [2600, 0, 2600, 100, 7], [-9, 2000, 500, 9999, 1300], [0, 2599, 1, 2598, 2600], [1500, 100, 2600, 1600, 1700]]


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def guarded(nbytes, fill):
    """(the whole allocation, the nbytes in its middle); the middle holds `fill`."""
    whole = torch.full((nbytes + 2 * PAD,), BYTE, dtype=torch.uint8, device="cuda")
    whole[PAD:PAD + nbytes] = fill
    return whole, whole[PAD:PAD + nbytes]


def untouched(whole):
    return bool((whole[:PAD] == BYTE).all()) and bool((whole[-PAD:] == BYTE).all())


@pytest.mark.parametrize("T,starts", [(100, s) for s in SMALL] + [(2600, s) for s in LARGE])
@pytest.mark.parametrize("prefixes", [None, [5, 99, -3, 5000]])
def test_rows_of_the_table(dh, T, starts, prefixes):
    """The kernels read rows between the first and the last row of any document, so no other row may be of one."""
    nbytes = dh.dh_docs_table_bytes(T, 2, 1)
    whole, table = guarded(nbytes, 0x5a)
    whole_pos, pos = guarded(4 * T, 0x5a)
    dh.dh_docs_plan(dh.docs(T, 4, 2, 1, i32(starts), None if prefixes is None else i32(prefixes), pos, table))
    torch.cuda.synchronize()
    assert untouched(whole) and untouched(whole_pos)
    words = table[:64 + 12 * T].view(torch.int32).cpu().long()  # a head of 16, then three a row (T is a multiple of 4)
    first, last = int(words[0]), int(words[1])
    lo, hi, pre = words[16:].view(3, T)
    r = torch.arange(T)
    assert 0 <= first <= last <= T
    mine = hi > lo
    assert bool(((first <= lo) & (lo <= r) & (r < hi) & (hi <= last) & (lo <= pre) & (pre <= hi))[mine].all())
    assert bool(((lo == r) & (hi == r) & (pre == r))[~mine].all())
    assert torch.equal(pos.view(torch.int32).cpu().long(), r - lo)


@pytest.mark.parametrize("dtype,d,cap", [("bf16", 128, 0.0), ("bf16", 128, 30.0), ("bf16", 64, 0.0), ("f32", 64, 0.0)])
@pytest.mark.parametrize("T,starts", [(100, s) for s in SMALL] + [(2600, s) for s in LARGE])
def test_nothing_around_the_buffers_is_written(dh, dtype, d, cap, T, starts):
    nq, nkv = 2, 1
    tt, dt = (torch.bfloat16, dh.DH_BF16) if dtype == "bf16" else (torch.float32, dh.DH_F32)
    size = 2 if dtype == "bf16" else 4
    g = torch.Generator().manual_seed(T + d)
    qkv, dout = torch.randn((T, 4 * d), generator=g).to(tt).cuda(), torch.randn((T, 2 * d), generator=g).to(tt).cuda()
    wsb = max(dh.dh_attn_docs_fwd_workspace_bytes(dt, T, nq, nkv, d), dh.dh_attn_docs_bwd_workspace_bytes(dt, T, nq, nkv, d), 16)
    sizes = dict(table=dh.dh_docs_table_bytes(T, nq, nkv), pos=4 * T, o=T * nq * d * size, lse=4 * nq * T, dqkv=T * 4 * d * size, delta=4 * nq * T, ws=wsb)
    b = {k: guarded(n, 0) for k, n in sizes.items()}
    docs = dh.docs(T, 4, nq, nkv, i32(starts), i32([5, 99, -3, 5000]), b["pos"][1], b["table"][1])
    dh.dh_docs_plan(docs)
    dh.dh_attn_docs_fwd(dt, docs, d, cap, qkv, b["o"][1], b["lse"][1], b["ws"][1], wsb)
    dh.dh_attn_docs_bwd(dt, docs, d, cap, qkv, b["o"][1], dout, b["lse"][1], b["dqkv"][1], b["delta"][1], b["ws"][1], wsb)
    torch.cuda.synchronize()
    assert [k for k in b if not untouched(b[k][0])] == []
    # rows of no document are left alone
    words = b["table"][1][64:64 + 8 * T].view(torch.int32).view(2, T)
    dead = words[0] == words[1]
    assert not bool(b["o"][1].view(T, -1)[dead].any()) and not bool(b["dqkv"][1].view(T, -1)[dead].any()) and not bool(b["lse"][1].view(torch.int32).view(nq, T)[:, dead].any())
