"""The norm of many gradient tensors and their clipping through the C ABI.  The norm is summed in float64 and rounded once (half a step, 2^-24, and 2^-40 for a sum of
up to 2^12 partial sums of float64 terms); a clipped element is one float32 product, rounded once more to its type, of a factor that is off by 2^-23."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def norm_of(dh, tensors, stream=None):
    lst = dh.tensor_list(tensors)
    wsb = dh.dh_grad_norm_ws_bytes(lst)
    norm, ws = torch.full((1,), -1.0, device="cuda"), torch.full((max(wsb, 8),), 0xff, dtype=torch.uint8, device="cuda")
    dh.dh_grad_norm(lst, norm, ws, wsb, stream)
    torch.cuda.synchronize()
    return norm


def exact(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


SIZES = {"one": [1], "few": [3, 0, 5], "odd": [1000, 1, 77, 65537, 8191, 0], "many": [1 + 37 * i % 1000 for i in range(300)], "chunks": [16384 * 5 + 3, 2048, 400000]}


@pytest.mark.parametrize("sizes", list(SIZES))
@pytest.mark.parametrize("types", ["f32", "bf16", "mixed"])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_norm_and_clip(dh, sizes, types, shift):
    g = torch.Generator().manual_seed(len(sizes) + shift)
    tensors, outs, wholes = [], [], []
    for i, n in enumerate(SIZES[sizes]):
        tt = torch.bfloat16 if types == "bf16" or (types == "mixed" and i % 2) else torch.float32
        whole = (torch.randn(n + 8, generator=g) * 10.0 ** (i % 5 - 3)).to(tt).cuda()
        wholes.append(torch.full((n + 8,), 3.0, dtype=tt, device="cuda"))
        tensors.append(whole[shift:shift + n])  # off their 16-byte boundaries, out by another offset
        outs.append(wholes[-1][(shift * 2) % 5:][:n])
    norm, want = norm_of(dh, tensors), exact(tensors)
    assert abs(float(norm) - want) <= (2.0 ** -24 + 2.0 ** -40) * 1.01 * want
    assert torch.equal(norm, norm_of(dh, tensors))
    for max_norm in (want * 0.37, want * 5):
        lst = dh.tensor_list(tensors, outs)
        before = [t.clone() for t in tensors]
        dh.dh_grad_clip(lst, norm, max_norm)
        torch.cuda.synchronize()
        f = min(1.0, max_norm / (want + 1e-6))
        for t, o, b, w in zip(tensors, outs, before, wholes):
            u = 2.0 ** -8 if t.dtype == torch.bfloat16 else 2.0 ** -24
            assert torch.equal(t, b)
            if f == 1.0:
                assert torch.equal(o, t)
            err = (1.01 * u + 4 * 2.0 ** -24) * (t.double() * f).abs() + 1e-40
            assert bool(((o.double() - t.double() * f).abs() <= err).all())
            assert int((w == 3.0).sum()) >= 8  # the elements around are as they were
        kept = [o.clone() for o in outs]
        dh.dh_grad_clip(dh.tensor_list(tensors), norm, max_norm)  # in place: the same bits
        torch.cuda.synchronize()
        assert all(torch.equal(t, k) for t, k in zip(tensors, kept))
        for t, b in zip(tensors, before):
            t.copy_(b)


def test_far_magnitudes(dh):
    """Squares beyond float32's range on both sides."""
    for scale in (1e30, 1e-30):
        t = [torch.full((1000,), scale, device="cuda"), torch.full((24,), -scale, device="cuda")]
        n = norm_of(dh, t)
        assert abs(float(n) - 32 * scale) <= 2.0 ** -22 * 32 * scale


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_norm_that_is_no_number_leaves_gradients(dh, value):
    t = torch.randn(5000, generator=torch.Generator().manual_seed(1)).cuda()
    t[4321] = value
    n = norm_of(dh, [t])
    assert not math.isfinite(float(n))
    before, out = t.clone(), torch.zeros_like(t)
    dh.dh_grad_clip(dh.tensor_list([t]), n, 0.5)
    dh.dh_grad_clip(dh.tensor_list([t], [out]), n, 0.5)
    torch.cuda.synchronize()
    assert torch.equal(t.view(torch.int32), before.view(torch.int32)) and torch.equal(out.view(torch.int32), before.view(torch.int32))


def test_nothing_has_norm_zero(dh):
    assert float(norm_of(dh, [])) == 0.0
    assert float(norm_of(dh, [torch.zeros(100, device="cuda")])) == 0.0
    dh.dh_grad_clip(dh.tensor_list([]), norm_of(dh, []), 1.0)


def test_replays(dh):
    """Norm and clipping captured, replayed on new gradients between eager runs: the same bits."""
    t = [torch.zeros(100001, device="cuda"), torch.zeros(70000, dtype=torch.bfloat16, device="cuda")]
    out = [torch.zeros_like(x) for x in t]
    lst = dh.tensor_list(t, out)
    wsb = dh.dh_grad_norm_ws_bytes(lst)
    ws, norm, s = torch.zeros(wsb, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda"), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())

    def step(stream):
        dh.dh_grad_norm(lst, norm, ws, wsb, stream)
        dh.dh_grad_clip(lst, norm, 1.0, stream)

    step(s)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s)
    for k in range(3):
        for x in t:
            x.copy_(torch.randn(x.shape, generator=torch.Generator().manual_seed(k)))
        torch.cuda.synchronize()
        step(s)
        s.synchronize()
        want = [norm.clone()] + [o.clone() for o in out]
        for o in out:
            o.zero_()
        norm.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([norm] + out, want))
