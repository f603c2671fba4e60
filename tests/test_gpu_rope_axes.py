"""Rotary positions from a table through the C ABI, against float64.  A result is a cos - b sin with both products and the sum rounded in float32 (3 w (|a| + |b|), w =
2^-24), an angle that is formed in float64, reduced, and rounded to float32 below pi (at most 2^-23 off) and sines of that (2 w), then one rounding to the storage type."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dh():
    from paper_2411_15871_amd import dhelix
    assert torch.cuda.is_available()
    return dhelix


def reference(x, pos, axes, n, d, base, pairing, form, inverse):
    x = x.double().view(x.shape[0], n, d)
    y, mag, first = torch.zeros_like(x), torch.zeros_like(x), 0
    for a, m in enumerate(axes):
        for i in range(first, first + m):
            w = pos[:, a].double() * base ** (-2.0 * i / d if form == 0 else -(i - first) / m)
            co, si = torch.cos(w)[:, None], torch.sin(w)[:, None] * (-1 if inverse else 1)
            u, v = (i, i + d // 2) if pairing == 0 else (2 * i, 2 * i + 1)
            y[:, :, u], y[:, :, v] = x[:, :, u] * co - x[:, :, v] * si, x[:, :, v] * co + x[:, :, u] * si
            mag[:, :, u] = mag[:, :, v] = x[:, :, u].abs() + x[:, :, v].abs()
        first += m
    return y.reshape(x.shape[0], -1), mag.reshape(x.shape[0], -1)


def close(got, want, mag, u):
    err = mag * (3 * 2.0 ** -24 + 2.0 ** -23 + 2 * 2.0 ** -24) + 1.01 * u * want.abs() + 1e-30
    bad = ~((got.double().cpu() - want).abs() <= err)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("T,heads,d,axes", [(1, 1, 16, (8,)), (7, 3, 64, (32,)), (130, 5, 128, (16, 24, 24)), (33, 2, 128, (1, 62, 1)), (40, 9, 80, (13, 20, 7)), (5, 1, 512, (100, 56, 99, 1)),
                                            (2000, 40, 128, (20, 44))])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pairing,form,inverse", [(0, 0, False), (1, 1, True), (0, 1, False), (1, 0, True)])
def test_axes(dh, dtype, T, heads, d, axes, pairing, form, inverse):
    tt, u = (torch.bfloat16, 2.0 ** -8) if dtype == "bf16" else (torch.float32, 2.0 ** -24)
    g = torch.Generator().manual_seed(T + d)
    x = torch.randn((T, heads * d + 24), generator=g).to(tt)
    pos = torch.randint(-1000, 1 << 20, (T, len(axes)), generator=g, dtype=torch.int32)
    pos[0] = 0
    want, mag = reference(x[:, :heads * d], pos, axes, heads, d, 10000.0, pairing, form, inverse)
    dt = dh.DH_BF16 if dtype == "bf16" else dh.DH_F32
    src, out = x.cuda(), torch.full((T, heads * d + 8), 5.0, dtype=tt, device="cuda")
    dh.dh_rope_axes(dt, pairing, form, T, axes, pos.cuda(), heads, d, 10000.0, inverse, src, heads * d + 24, out, heads * d + 8)
    torch.cuda.synchronize()
    close(out[:, :heads * d], want, mag, u)
    assert bool((out[:, heads * d:] == 5.0).all()) and torch.equal(src.cpu(), x)
    # in place: the same bits, what lies behind the heads as it was
    dh.dh_rope_axes(dt, pairing, form, T, axes, pos.cuda(), heads, d, 10000.0, inverse, src, heads * d + 24, src, heads * d + 24)
    torch.cuda.synchronize()
    assert torch.equal(src[:, :heads * d], out[:, :heads * d]) and torch.equal(src.cpu()[:, heads * d:], x[:, heads * d:])


def test_one_axis_is_the_plain_rotation(dh):
    """Positions 0, 1, 2 ... on one axis: the operator for equal sequences, up to its own rounding of the frequencies."""
    T, heads, d = 300, 4, 128
    x = torch.randn((T, heads * d), generator=torch.Generator().manual_seed(1)).cuda()
    a, b, back = x.clone(), torch.empty_like(x), torch.empty_like(x)
    dh.dh_rope(dh.DH_F32, T, 100, heads, d, heads * d, 10000.0, False, a)
    pos = (torch.arange(T, dtype=torch.int32) % 100).cuda()
    dh.dh_rope_axes(dh.DH_F32, 0, 0, T, (d // 2,), pos, heads, d, 10000.0, False, x, heads * d, b, heads * d)
    dh.dh_rope_axes(dh.DH_F32, 0, 0, T, (d // 2,), pos, heads, d, 10000.0, True, b, heads * d, back, heads * d)
    torch.cuda.synchronize()
    size = float(x.abs().max())
    assert float((a - b).abs().max()) <= 2 * 2 * size * 8 * 2.0 ** -24  # two results, each off by 8 w (|a| + |b|)
    assert float((back - x).abs().max()) <= 2 * 2 * size * 8 * 2.0 ** -24 * 1.5  # there and back: the second turn carries the first's error


@pytest.mark.parametrize("value", [2 ** 31 - 1, -2 ** 31])
def test_largest_positions(dh, value):
    x = torch.randn((3, 64), generator=torch.Generator().manual_seed(2))
    pos = torch.tensor([[value], [value // 2], [value // 3]], dtype=torch.int32)
    out = torch.empty((3, 64), device="cuda")
    dh.dh_rope_axes(dh.DH_F32, 0, 0, 3, (32,), pos.cuda(), 1, 64, 10000.0, False, x.cuda(), 64, out, 64)
    want, mag = reference(x, pos, (32,), 1, 64, 10000.0, 0, 0, False)
    torch.cuda.synchronize()
    # an angle of 2^31 in float64 is off by 2^-22 for its own rounding and 2 more for its frequency's
    err = mag * (8 * 2.0 ** -24 + 3 * 2.0 ** -22) + 2.0 ** -24 * want.abs()
    assert bool(((out.double().cpu() - want).abs() <= err).all())
