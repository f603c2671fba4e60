"""What window attention, linear attention and dropout refuse, before anything is launched.  No GPU needed: the addresses are never read."""
import pytest

from paper_2411_15871_amd import dhelix as dh

A, BIG = 1 << 20, 1 << 50  # an aligned address that nobody reads; room enough
INVALID, SHAPE, SMALL = dh.DH_ERR_INVALID_ARG, dh.DH_ERR_SHAPE, dh.DH_ERR_WORKSPACE_TOO_SMALL


def refused(code, fn, *args):
    with pytest.raises(dh.DhelixError) as e:
        fn(*args)
    assert e.value.code == code, str(e.value)


def pointers(n, i, bad):
    p = [A] * n
    p[i] = bad
    return p


SIZES = dict(dtype=dh.DH_BF16, batch=2, seq=100, window=10, sinks=2, nq=4, nkv=2, d=128)
BAD_SIZES = [(dict(dtype=9), INVALID), (dict(batch=-1), SHAPE), (dict(seq=-1), SHAPE), (dict(nq=0), SHAPE), (dict(nkv=0), SHAPE), (dict(nkv=3), SHAPE), (dict(nq=1026), SHAPE), (dict(d=96), SHAPE),
             (dict(d=256), SHAPE), (dict(dtype=dh.DH_F32, d=4), SHAPE), (dict(dtype=dh.DH_F32, d=136), SHAPE), (dict(dtype=dh.DH_F32, d=0), SHAPE), (dict(batch=65536), SHAPE),
             (dict(seq=(1 << 26) + 1), SHAPE), (dict(batch=60000, seq=1 << 20), SHAPE)]


@pytest.mark.parametrize("bad,code", BAD_SIZES + [(dict(window=0), SHAPE), (dict(window=-5), SHAPE), (dict(sinks=-1), SHAPE)])
def test_window_sizes(bad, code):
    s = list({**SIZES, **bad}.values())
    refused(code, dh.dh_attn_window_fwd, *s, A, A, A, A, BIG)
    refused(code, dh.dh_attn_window_bwd, *s, A, A, A, A, A, A, A, BIG)
    if "seq" not in bad:
        s[2], s[3], s[4] = 64, s[3], s[4]
        refused(code, dh.dh_attn_window_step, *s, A, A, A, A, A, BIG)


def test_window_pointers():
    s = list(SIZES.values())
    for i in range(3):
        refused(INVALID, dh.dh_attn_window_fwd, *s, *pointers(3, i, None), A, BIG)
        if i < 2:
            refused(INVALID, dh.dh_attn_window_fwd, *s, *pointers(3, i, A + 8), A, BIG)
    for i in range(6):
        refused(INVALID, dh.dh_attn_window_bwd, *s, *pointers(6, i, None), A, BIG)
        if i in (0, 1, 2, 4):
            refused(INVALID, dh.dh_attn_window_bwd, *s, *pointers(6, i, A + 8), A, BIG)
    for fn, size, n in ((dh.dh_attn_window_fwd, dh.dh_attn_window_fwd_workspace_bytes, 3), (dh.dh_attn_window_bwd, dh.dh_attn_window_bwd_workspace_bytes, 6)):
        refused(INVALID, fn, *s, *[A] * n, A + 8, BIG)
        for sizes in (s, [dh.DH_BF16, 1, 4096, 512, 4, 4, 1, 128]):
            need = size(*sizes)
            if need:
                refused(SMALL, fn, *sizes, *[A] * n, A, need - 1)
                refused(SMALL, fn, *sizes, *[A] * n, None, need)


def test_window_step():
    s = [dh.DH_BF16, 2, 12, 10, 2, 4, 2, 128]
    for i in range(4):
        refused(INVALID, dh.dh_attn_window_step, *s, *pointers(4, i, None), A, BIG)
        refused(INVALID, dh.dh_attn_window_step, *s, *pointers(4, i, A + 2), A, BIG)
    refused(INVALID, dh.dh_attn_window_step, *s, *[A] * 4, A + 8, BIG)
    for rows, window, sinks in ((11, 10, 2), (0, 1, 0), (-4, 1, 0), (2 ** 31 - 1, 2 ** 31 - 1, 1)):
        refused(SHAPE, dh.dh_attn_window_step, dh.DH_BF16, 2, rows, window, sinks, 4, 2, 128, A, A, A, A, A, BIG)
    refused(SHAPE, dh.dh_attn_window_step, dh.DH_BF16, 2, 2 ** 30 + 1, 1024, 4, 4, 2, 128, A, A, A, A, A, BIG)
    need = dh.dh_attn_window_step_workspace_bytes(dh.DH_BF16, 1, 8192, 4096, 4, 4, 1, 128)
    assert need > 0
    refused(SMALL, dh.dh_attn_window_step, dh.DH_BF16, 1, 8192, 4096, 4, 4, 1, 128, A, A, A, A, A, need - 1)


@pytest.mark.parametrize("bad,code", BAD_SIZES)
def test_linear_sizes(bad, code):
    s = {**SIZES, **bad}
    s = [s[k] for k in ("dtype", "batch", "seq", "nq", "nkv", "d")] + [1.0]
    refused(code, dh.dh_linattn_fwd, *s, A, A, None, A, None, A, BIG)
    refused(code, dh.dh_linattn_bwd, *s, A, A, None, A, None, A, None, A, BIG)
    if "seq" not in bad:
        refused(code, dh.dh_linattn_step, *s[:2], *s[3:], A, None, A, A, A, A)


def test_linear_pointers():
    s = [dh.DH_BF16, 2, 100, 4, 2, 128, 1.0]
    bytes_ = 2 * 2 * 128 * 128 * 4
    far = A + bytes_
    for i, may in ((0, False), (1, False), (2, True), (3, False), (4, True)):  # log_decay, qkv, state_in, o, state_out
        p = [A, A, A, A, far]
        p[i] = A + 2 if i == 0 else A + 8 + (bytes_ if i == 4 else 0)
        refused(INVALID, dh.dh_linattn_fwd, *s, *p, A, BIG)
        if not may:
            p[i] = None
            refused(INVALID, dh.dh_linattn_fwd, *s, *p, A, BIG)
    refused(INVALID, dh.dh_linattn_fwd, *s, A, A, A, A, far - 16, A, BIG)
    refused(INVALID, dh.dh_linattn_fwd, *s, A, A, A, A, A, A, BIG)
    for i, may in ((0, False), (1, False), (2, True), (3, False), (4, True), (5, False), (6, True)):  # log_decay, qkv, state_in, dout, dstate_out, dqkv, dstate_in
        p = [A, A, A, A, A, A, far]
        p[i] = A + 2 if i == 0 else p[i] + 8
        refused(INVALID, dh.dh_linattn_bwd, *s, *p, A, BIG)
        if not may:
            p[i] = None
            refused(INVALID, dh.dh_linattn_bwd, *s, *p, A, BIG)
    refused(INVALID, dh.dh_linattn_bwd, *s, A, A, A, A, A, A, far - 16, A, BIG)
    for fn, size, p in ((dh.dh_linattn_fwd, dh.dh_linattn_fwd_workspace_bytes, [A, A, None, A, None]), (dh.dh_linattn_bwd, dh.dh_linattn_bwd_workspace_bytes, [A, A, None, A, None, A, None])):
        refused(INVALID, fn, *s, *p, A + 8, BIG)
        sizes = [dh.DH_BF16, 1, 4096, 4, 1, 128]
        need = size(*sizes)
        if need:
            refused(SMALL, fn, *sizes, 1.0, *p, A, need - 1)
            refused(SMALL, fn, *sizes, 1.0, *p, None, need)


def test_linear_step():
    s = [dh.DH_BF16, 2, 4, 2, 128, 1.0]
    for i in range(6):  # log_decay, pos, qkv, state_in, state_out, o
        p = pointers(6, i, A + 2)
        refused(INVALID, dh.dh_linattn_step, *s, *p)
        if i != 1:
            refused(INVALID, dh.dh_linattn_step, *s, *pointers(6, i, None))
    refused(INVALID, dh.dh_linattn_step, *s, A, None, A, A, A + 1024, A)


def test_dropout():
    def fwd(code, dtype=dh.DH_BF16, T=4, H=64, a=A, b=A, bias=A, p=0.1, rng=A, out=A):
        refused(code, dh.dh_dropout_add_fwd, dtype, T, H, a, b, bias, p, rng, 0, out)

    def bwd(code, dtype=dh.DH_BF16, T=4, H=64, dout=A, p=0.1, rng=A, dx=A, dbias=A, ws=A, n=BIG):
        refused(code, dh.dh_dropout_add_bwd, dtype, T, H, dout, p, rng, 0, dx, dbias, False, ws, n)

    for f in (fwd, bwd):
        f(INVALID, dtype=4)
        for H in (0, -8, 12):
            f(SHAPE, H=H)
        f(SHAPE, T=-1)
        for p in (-0.1, 1.01, float("nan"), float("inf")):
            f(INVALID, p=p)
        f(INVALID, rng=None)
        f(INVALID, rng=A + 4)
    for k in ("a", "b", "bias", "out"):
        fwd(INVALID, **{k: A + 8})
    for k in ("b", "out"):
        fwd(INVALID, **{k: None})
    for k in ("dout", "dx"):
        bwd(INVALID, **{k: A + 8})
        bwd(INVALID, **{k: None})
    bwd(INVALID, dbias=A + 2)
    bwd(INVALID, ws=A + 8)
    need = dh.dh_dropout_add_bwd_ws_bytes(4096, 64)
    bwd(SMALL, T=4096, n=need - 1)
    bwd(SMALL, T=4096, ws=None)


def test_nothing_to_do_is_no_error():
    for t in (dh.DH_BF16, dh.DH_F32):
        for batch, seq in ((0, 5), (2, 0)):
            dh.dh_attn_window_fwd(t, batch, seq, 1, 0, 2, 1, 64, None, None, None)
            dh.dh_attn_window_bwd(t, batch, seq, 1, 0, 2, 1, 64, None, None, None, None, None, None)
        dh.dh_attn_window_step(t, 0, 8, 4, 0, 2, 1, 64, None, None, None, None)
        dh.dh_linattn_fwd(t, 0, 5, 2, 1, 64, 1.0, None, None, None, None, None)
        dh.dh_linattn_bwd(t, 0, 5, 2, 1, 64, 1.0, None, None, None, None, None, None, None)
        dh.dh_linattn_step(t, 0, 2, 1, 64, 1.0, None, None, None, None, None, None)
        dh.dh_dropout_add_fwd(t, 0, 64, None, None, None, 0.5, None, 0, None)
        dh.dh_dropout_add_bwd(t, 0, 64, None, 0.5, None, 0, None, None, False)
    for size in (dh.dh_linattn_fwd_workspace_bytes, dh.dh_linattn_bwd_workspace_bytes):
        assert size(dh.DH_BF16, 1, 0, 2, 1, 64) == 0 and size(dh.DH_BF16, 1, 100, 3, 2, 64) == 0 and size(7, 1, 100, 2, 1, 64) == 0
    assert dh.dh_dropout_add_bwd_ws_bytes(0, 64) == 0 and dh.dh_attn_window_step_workspace_bytes(dh.DH_BF16, 1, 8, 0, 0, 2, 1, 64) == 0
