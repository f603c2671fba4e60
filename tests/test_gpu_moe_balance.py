"""Balance loss, z loss and counts of the router through the C ABI, against float64.  A softmax over E terms in float32 is off by (E + 24) w relatively (w = 2^-24: the
terms' sum, the exponentials of differences up to 2 w |logit| away, the quotient), a sum over N tokens by N w of its terms at most."""
import pytest
import torch

pytestmark = pytest.mark.gpu
W = 2.0 ** -24


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def reference(logits, idx, N, dloss):
    T, E = logits.shape
    z = logits[:N].double()
    L = torch.logsumexp(z, 1) if N else torch.zeros(0).double()
    some = torch.isfinite(L) if N else torch.zeros(0, dtype=torch.bool)
    p = torch.where(some[:, None], torch.exp(z - torch.where(some, L, torch.zeros(()).double())[:, None]), torch.zeros(()).double())
    counts = torch.bincount(idx[:N].reshape(-1).long(), minlength=E)
    n = max(N, 1)
    f, mean = counts.double() / (2 * n), p.sum(0) / n
    Lz = torch.where(some, L, torch.zeros(()).double())
    d = torch.zeros((T, E)).double()
    d[:N] = p * (dloss[0].double() * E / n * (f - (p * f).sum(1, keepdim=True)) + dloss[1].double() * 2 / n * Lz[:, None])
    size = torch.zeros((T, E)).double()
    size[:N] = p * (dloss[0].abs().double() * E / n * (f + (p * f).sum(1, keepdim=True)) + dloss[1].abs().double() * 2 / n * Lz.abs()[:, None])
    return counts, mean, L, torch.stack([E * (f * mean).sum(), (Lz * Lz).sum() / n]), d, size


def run(dh, T, E, pad, seed, logits=None, n_live=True, accumulate=False):
    g = torch.Generator().manual_seed(seed)
    logits = torch.randn((T, E), generator=g) * 2 + torch.randn(E, generator=g) if logits is None else logits
    idx = torch.empty((T, 2), dtype=torch.int32, device="cuda")
    prob = torch.empty((T, 2), device="cuda")
    lg = logits.cuda()
    dh.dh_moe_route(T, E, lg, idx, prob)
    N = T - pad
    live = torch.tensor([N], dtype=torch.int32, device="cuda") if n_live else None
    dloss = torch.tensor([0.7, -0.3])
    counts, mean = torch.full((E,), -5, dtype=torch.int32, device="cuda"), torch.full((E,), 9.0, device="cuda")
    lse, loss = torch.full((T,), 7.0, device="cuda"), torch.full((2,), 9.0, device="cuda")
    before = torch.randn((T, E), generator=g)
    dlogits = before.cuda() if accumulate else torch.full((T, E), 5.0, device="cuda")
    wsb = dh.dh_moe_balance_ws_bytes(T, E)
    ws = torch.full((wsb,), 0xff, dtype=torch.uint8, device="cuda")
    dh.dh_moe_balance_fwd(T, E, lg, idx, live, counts, mean, lse, loss, ws, wsb)
    dh.dh_moe_balance_bwd(T, E, lg, lse, counts, live, dloss.cuda(), accumulate, dlogits)
    torch.cuda.synchronize()
    N = min(max(N, 0), T)
    c, m, L, l, d, size = reference(logits, idx.cpu(), N, dloss)
    assert torch.equal(counts.cpu().long(), c)
    far = float(logits[torch.isfinite(logits)].abs().max()) if torch.isfinite(logits).any() else 0.0
    rel = (E + 24 + 4 * far) * W
    assert bool(((mean.cpu().double() - m).abs() <= (rel + (N + 4) * W) * m + 1e-30).all())
    got = lse.cpu().double()
    some = torch.isfinite(L)
    assert bool(((got[:N][some] - L[some]).abs() <= rel + 2 * W * L[some].abs()).all()) and bool((got[:N][~some] == L[~some]).all()) and bool((got[N:] == 7.0).all())
    big = float(L[some].abs().max()) if some.any() else 0.0
    assert abs(float(loss[0]) - float(l[0])) <= (rel + (N + E + 8) * W) * float(l[0]) + 1e-30
    assert abs(float(loss[1]) - float(l[1])) <= (N + 8) * W * float(l[1]) + 2 * rel * big + 1e-30
    out = dlogits.cpu().double()
    err = (2 * rel + (E + 16) * W) * size + (W * (out.abs() + before.abs().double()) if accumulate else 0.0) + 1e-30
    want = d + before.double() if accumulate else d
    assert bool(((out - want).abs() <= err).all())
    if accumulate:
        assert torch.equal(dlogits.cpu()[N:], before[N:])
    return loss


@pytest.mark.parametrize("T,E,pad", [(1, 2, 0), (2, 3, 1), (7, 5, 0), (64, 8, 3), (100, 16, 0), (333, 17, 33), (513, 64, 0), (200, 65, 7), (300, 128, 0), (1000, 200, 10), (77, 256, 0),
                                     (5000, 16, 1)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_sizes(dh, T, E, pad, accumulate):
    run(dh, T, E, pad, T + E, accumulate=accumulate)


def test_all_live_and_none(dh):
    run(dh, 50, 16, 0, 1, n_live=False)
    run(dh, 50, 16, 50, 2)   # no token counts
    run(dh, 50, 16, 60, 3)   # a negative count: none
    run(dh, 50, 16, -20, 4)  # more than there are: all


def test_balanced_router_has_loss_one(dh):
    """Equal logits moved by hair: every expert as likely as another, counts as the router breaks ties."""
    loss = run(dh, 64, 8, 0, 5, logits=torch.zeros((64, 8)))
    assert abs(float(loss[0]) - 1.0) <= 64 * W  # E sum f / E = sum f = 1


def test_masked_logits(dh):
    """Minus infinity and the type's lowest value as masks, also of whole tokens."""
    logits = torch.randn((40, 12), generator=torch.Generator().manual_seed(6))
    logits[:, 3] = float("-inf")
    logits[5] = float("-inf")
    logits[7, 1:] = float("-inf")
    run(dh, 40, 12, 2, 7, logits=logits)
    low = torch.randn((40, 12), generator=torch.Generator().manual_seed(8)).clamp(-3, 3)
    low[:, 4:] = torch.finfo(torch.float32).min
    lg = low.clone()
    T, E = lg.shape
    idx = torch.zeros((T, 2), dtype=torch.int32, device="cuda")
    prob, x = torch.zeros((T, 2), device="cuda"), lg.cuda()
    counts, mean, lse, loss = torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(E, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(2, device="cuda")
    dh.dh_moe_route(T, E, x, idx, prob)
    wsb = dh.dh_moe_balance_ws_bytes(T, E)
    dh.dh_moe_balance_fwd(T, E, x, idx, None, counts, mean, lse, loss, torch.zeros(wsb, dtype=torch.uint8, device="cuda"), wsb)
    torch.cuda.synchronize()
    assert bool((mean[4:] == 0).all()) and abs(float(mean.sum()) - 1.0) <= 64 * W and bool(torch.isfinite(loss).all())


def test_gradient_against_differences(dh):
    T, E, N = 30, 6, 28
    g = torch.Generator().manual_seed(9)
    logits, direction = torch.randn((T, E), generator=g), torch.randn((T, E), generator=g).double()
    idx = torch.topk(logits, 2, dim=1).indices.to(torch.int32)
    dloss = torch.tensor([1.0, 0.5])

    def value(step):  # counts are constants
        _, _, _, l, _, _ = reference((logits.double() + step * direction), idx, N, dloss)
        return float((l * dloss.double()).sum())

    x, lse, dl = logits.cuda(), torch.zeros(T, device="cuda"), torch.zeros((T, E), device="cuda")
    counts, mean, loss = torch.zeros(E, dtype=torch.int32, device="cuda"), torch.zeros(E, device="cuda"), torch.zeros(2, device="cuda")
    live, wsb = torch.tensor([N], dtype=torch.int32, device="cuda"), dh.dh_moe_balance_ws_bytes(T, E)
    dh.dh_moe_balance_fwd(T, E, x, idx.cuda(), live, counts, mean, lse, loss, torch.zeros(wsb, dtype=torch.uint8, device="cuda"), wsb)
    dh.dh_moe_balance_bwd(T, E, x, lse, counts, live, dloss.cuda(), False, dl)
    torch.cuda.synchronize()
    want = (value(1e-5) - value(-1e-5)) / 2e-5
    assert abs(float((dl.cpu().double() * direction).sum()) - want) <= 1e-5 * float((dl.cpu().double() * direction).abs().sum())
