"""How many bits the router's balance loss keeps (w = 2^-24, half a step of float32).  Logits are multiples of 1/16, so that differences of them are exact.  A probability exp(x) / sum: an
exponential is off by 3 w and 2^-29 |x| log2(e), that is 7 w for x down to -80; a sum of E <= 256 of them by that and, added by lanes of four, in at most 9 roundings more; the quotient and the product round
once each: 25 w.  None of it grows with the number of tokens."""
import pytest
import torch

pytestmark = pytest.mark.gpu
W = 2.0 ** -24


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    yield dhelix
    torch.cuda.empty_cache()


def both(dh, x, dloss):
    T, E = x.shape
    idx = torch.arange(2, dtype=torch.int32, device="cuda").repeat(T, 1)
    counts, mean = torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(E, device="cuda")
    lse, loss, dl = torch.zeros(T, device="cuda"), torch.zeros(2, device="cuda"), torch.empty((T, E), device="cuda")
    wsb = dh.dh_moe_balance_ws_bytes(T, E)
    ws = torch.empty(wsb, dtype=torch.uint8, device="cuda")
    dh.dh_moe_balance_fwd(T, E, x, idx, None, counts, mean, lse, loss, ws, wsb)
    dh.dh_moe_balance_bwd(T, E, x, lse, counts, None, torch.tensor(dloss, device="cuda"), False, dl)
    torch.cuda.synchronize()
    return mean.double().cpu(), lse.double().cpu(), loss.double().cpu(), dl


@pytest.mark.parametrize("E", [256, 255, 64, 61, 8])
@pytest.mark.parametrize("lowest", [-8.0, -80.0])
def test_small_probabilities(dh, E, lowest):
    """One token: prob_mean is its softmax, the z loss's gradient 2 lse p."""
    x = (torch.linspace(0, lowest, E) * 16).round() / 16
    x = x[torch.randperm(E, generator=torch.Generator().manual_seed(E))]
    mean, lse, loss, dl = both(dh, x[None].cuda(), [0.0, 1.0])
    L, p = torch.logsumexp(x.double(), 0), torch.softmax(x.double(), 0)
    assert float(((mean - p).abs() / p).max()) <= 25 * W
    assert abs(float(lse[0] - L)) <= 16 * W + 3 * W * float(L)  # the sum's error, the logarithm's and its rounding
    want = 2 * L * p
    assert float(((dl[0].double().cpu() - want).abs() / want).max()) <= (25 + 16 / float(L) + 3 + 4) * W


@pytest.mark.parametrize("T,E", [(1 << 20, 256), (1 << 20, 255), (1 << 22, 8), (300000, 3)])
def test_many_equal_tokens(dh, T, E):
    """The same logits in every row, whose roundings would all go one way in a float32 sum: means off by 25 w, three roundings of four tokens' sum, seven of a wave's (its lanes' sums and up to six
    steps across them), four of 16 waves' in pairs, and three of all blocks' and the mean."""
    x = (torch.randn(E, generator=torch.Generator().manual_seed(E)).clamp(-3, 3) * 16).round() / 16
    mean, lse, loss, dl = both(dh, x.cuda().repeat(T, 1), [1.0, 0.0])
    L, p = torch.logsumexp(x.double(), 0), torch.softmax(x.double(), 0)
    assert float(((mean - p).abs() / p).max()) <= 42 * W
    assert abs(float(loss[1] - L * L)) <= 2 * (16 * W + 4 * W * float(L)) * float(L) + 19 * W * float(L * L)
    assert abs(float(loss[0]) - float(E * (p[0] + p[1]) / 2)) <= (42 + 12) * W * float(E * (p[0] + p[1]) / 2)
