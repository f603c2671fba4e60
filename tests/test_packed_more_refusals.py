"""More of what the operators of packed micro-batches refuse, before anything is launched.  No GPU needed: the addresses are never read."""
import pytest
import torch

from paper_2411_15871_amd import dhelix as dh
from test_packed_refusals import A, docs, refused


@pytest.mark.parametrize("n", [(1 << 28) + 1, 1 << 30, (1 << 31) - 1])
def test_more_documents_than_the_plan_searches(n):
    """A search among n starts adds two places: from 2^30 on that passes 32 bits."""
    big = 1 << 40
    refused(dh.DH_ERR_SHAPE, dh.dh_docs_plan, docs(n_docs=n))
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_fwd, dh.DH_BF16, docs(n_docs=n), 128, 0.0, A, A, A, A, big)
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_bwd, dh.DH_BF16, docs(n_docs=n), 128, 0.0, A, A, A, A, A, A, A, big)


@pytest.mark.parametrize("T,nq,nkv", [(1, 1, 1), (100, 4, 2), (5000, 32, 8), (1 << 20, 8, 1)])
def test_a_table_that_is_too_short(T, nq, nkv):
    need, big, size = dh.dh_docs_table_bytes(T, nq, nkv), 1 << 60, dict(T=T, nq=nq, nkv=nkv)
    fwd, bwd = (dh.DH_BF16, docs(**size, table_bytes=0), 128, 0.0, A, A, A, A, big), (dh.DH_BF16, docs(**size, table_bytes=need - 1), 128, 0.0, A, A, A, A, A, A, A, big)
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_docs_plan, docs(**size, table_bytes=need - 1))
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_attn_docs_fwd, *fwd)
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_attn_docs_bwd, *bwd)
    for cut in (1, 16, 64 + 12 * T // 2):  # the forward pass reads a head, three ints a row and its own list
        refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_attn_docs_fwd, dh.DH_BF16, docs(**size, table_bytes=64 + 12 * T - cut if cut < 64 + 12 * T else 0), 128, 0.0, A, A, A, A, big)


def test_bytes_of_a_tensor():
    for dtype in (torch.uint8, torch.int32):
        t = torch.empty(48, dtype=dtype)
        assert dh.docs(100, 3, 4, 2, A, None, None, t).table_bytes == t.numel() * t.element_size()
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_docs_plan, dh.docs(100, 3, 4, 2, A, None, None, torch.empty(64, dtype=torch.int32)))
    assert docs().table_bytes == dh.dh_docs_table_bytes(100, 4, 2)
