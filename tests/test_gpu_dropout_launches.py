"""Dropout's backward pass with the bias gradient in two launches (more rows, or more elements, than one block for 32 columns takes): both types, ragged column and row groups, sums that are
added to, and sizes at the ends of 32 bits."""
import pytest
import torch

import mixers_ref as R
from test_gpu_dropout import BF, F, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


@pytest.mark.parametrize("T,H", [(2049, 24), (2500, 520), (4099, 8), (2064, 1032)])
@pytest.mark.parametrize("tt", [BF, F])
def test_two_launches(dh, tt, T, H):
    c = Case(dh, tt, T, H, 0.3)
    assert c.wsb > 0
    c.forward()
    c.backward()
    c.check()
    c.dbias.fill_(2.0)
    before = c.dbias.clone()
    c.dx.fill_(3.0)
    c.ws.fill_(0xff)
    c.backward(accumulate=True)
    c.check(before)
    c.dx = c.dout_d  # in place
    c.backward()
    c.check()


def test_the_last_number_of_rows(dh):
    """2^31 - 1 rows of one vector, 32 GiB: shared out as any others, the last one's bits those of its counter."""
    T, H = 2 ** 31 - 1, 8
    x = torch.ones((T, H), dtype=BF, device="cuda")
    rng = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
    n = dh.dh_dropout_add_bwd_ws_bytes(T, H)
    ws, dbias = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda"), torch.zeros(H, device="cuda")
    dh.dh_dropout_add_bwd(dh.DH_BF16, T, H, x, 0.5, rng, 1, x, dbias, False, ws, n)
    for v in (0, 12345, 2 ** 30, T - 2, T - 1):
        want = [0.0 if b < 32768 else 2.0 for w in R.philox([v & 0xFFFFFFFF, v >> 32, 6, 1], [5, 0]) for b in (w & 0xFFFF, w >> 16)]
        assert x[v].tolist() == want
    total = torch.zeros(H, dtype=torch.float64, device="cuda")
    for r in range(0, T, 2 ** 26):
        total += x[r:r + 2 ** 26].sum(0, dtype=torch.float64)
    # each block's sums are whole numbers below 2^24: exact; then 2048 of them, 256 in a row by eight threads, and these
    assert ((dbias.double() - total).abs() <= 264 * R.W * total).all()


def test_the_last_number_of_columns(dh):
    """2^29 columns have more threads than a launch counts along an axis; 2^31 - 8 are the last that there are."""
    H = 2 ** 29
    x = torch.ones((1, H), dtype=BF, device="cuda")
    rng = torch.tensor([5, 6], dtype=torch.int64, device="cuda")
    n = dh.dh_dropout_add_bwd_ws_bytes(1, H)
    ws, dbias = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda"), torch.full((H,), 3.0, device="cuda")
    dh.dh_dropout_add_bwd(dh.DH_BF16, 1, H, x, 0.5, rng, 1, x, dbias, True, ws, n)
    v = H // 8 - 1
    assert x[0, -8:].tolist() == [0.0 if b < 32768 else 2.0 for w in R.philox([v, 0, 6, 1], [5, 0]) for b in (w & 0xFFFF, w >> 16)]
    assert torch.equal(dbias, 3.0 + x[0].float())
    del x, ws, dbias
    H = 2 ** 31 - 8
    dbias = torch.full((H,), 3.0, device="cuda")
    dh.dh_dropout_add_bwd(dh.DH_BF16, 0, H, None, 0.5, None, 1, None, dbias, False, None, 0)
    assert not dbias.any()
