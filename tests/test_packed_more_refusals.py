"""More of what the operators of packed micro-batches refuse, before anything is launched.  No GPU needed: the addresses are never read."""
import pytest

from paper_2411_15871_amd import dhelix as dh
from test_packed_refusals import A, docs, refused


@pytest.mark.parametrize("n", [(1 << 28) + 1, 1 << 30, (1 << 31) - 1])
def test_more_documents_than_the_plan_searches(n):
    """A search among n starts adds two places: from 2^30 on that passes 32 bits."""
    big = 1 << 40
    refused(dh.DH_ERR_SHAPE, dh.dh_docs_plan, docs(n_docs=n))
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_fwd, dh.DH_BF16, docs(n_docs=n), 128, 0.0, A, A, A, A, big)
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_bwd, dh.DH_BF16, docs(n_docs=n), 128, 0.0, A, A, A, A, A, A, A, big)
