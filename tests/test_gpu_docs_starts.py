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


def table_of(dh, T, starts):
    table, pos = torch.empty(dh.dh_docs_table_bytes(T, 2, 1), dtype=torch.uint8, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
    start = torch.as_tensor(starts, dtype=torch.int32).cuda()
    docs = dh.docs(T, len(starts) - 1, 2, 1, start, None, pos, table)
    docs.keep = (table, pos, start)
    return docs


@pytest.mark.parametrize("T,places", [(1000, {0: 1, 5: 300, 70: 64, 130: 63, 131: 65, 200: 1, 700: 5000, 900: 1}), (1000, {0: 70000, 1: 64, 2: 128, 3: 1, 63: 200, 64: 200, 65: 200, 990: 100000}),
                                      (1000, {10: 1, 11: 4097, 1000: 9000}), (64, {3: 64, 40: 1000})])
def test_many_empty_documents(dh, T, places):
    """places: row -> how many documents begin there; all but the last of them are empty."""
    starts = [r for r, n in sorted(places.items()) for _ in range(n)]
    docs = table_of(dh, T, starts)
    dh.dh_docs_plan(docs)
    torch.cuda.synchronize()
    table, pos, _ = docs.keep
    words = table[:64 + 12 * T].view(torch.int32).cpu().long()
    lo, hi, pre = words[16:].view(3, T)
    rows = sorted(places)
    want_lo, want_hi = torch.arange(T), torch.arange(T)
    for a, z in zip(rows, rows[1:]):
        want_lo[a:z], want_hi[a:z] = a, z
    assert torch.equal(lo, want_lo) and torch.equal(hi, want_hi) and torch.equal(pre, want_lo) and torch.equal(pos.cpu().long(), torch.arange(T) - want_lo)


@pytest.mark.parametrize("n", [4000, 1 << 20])
def test_starts_padded_to_a_capacity(dh, n):
    """Starts behind the last document, all at its end: a micro-batch of few documents takes little longer to plan (one by one, a million starts took 2700 times as long)."""
    T, few = 8192, [0, 900, 4000, 8100]
    plain, padded = table_of(dh, T, few), table_of(dh, T, few + [8100] * (n - len(few)))

    def microseconds(docs):
        best = float("inf")
        for _ in range(5):
            dh.dh_docs_plan(docs)
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(5):
                dh.dh_docs_plan(docs)
            b.record()
            b.synchronize()
            best = min(best, a.elapsed_time(b) * 200)
        return best

    assert microseconds(padded) <= 8 * microseconds(plain)
