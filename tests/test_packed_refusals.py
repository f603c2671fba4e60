"""What the operators of packed micro-batches refuse, before anything is launched.  No GPU needed: the addresses are never read."""
import ctypes as C

import pytest

from paper_2411_15871_amd import dhelix as dh

A = 1 << 20  # an aligned address that nobody reads


def docs(**kw):
    f = dict(T=100, n_docs=3, nq=4, nkv=2, doc_start=A, prefix=None, pos=None, table=A)
    f.update(kw)
    return dh.docs(**f)


def refused(code, fn, *args, **kw):
    with pytest.raises(dh.DhelixError) as e:
        fn(*args, **kw)
    assert e.value.code == code, str(e.value)


@pytest.mark.parametrize("bad,code", [(dict(T=-1), dh.DH_ERR_SHAPE), (dict(n_docs=-1), dh.DH_ERR_SHAPE), (dict(nq=0), dh.DH_ERR_SHAPE), (dict(nkv=0), dh.DH_ERR_SHAPE),
                                      (dict(nkv=3), dh.DH_ERR_SHAPE), (dict(doc_start=None), dh.DH_ERR_INVALID_ARG), (dict(table=None), dh.DH_ERR_INVALID_ARG),
                                      (dict(table=A + 8), dh.DH_ERR_INVALID_ARG), (dict(T=(1 << 28) + 1), dh.DH_ERR_SHAPE), (dict(nq=1026), dh.DH_ERR_SHAPE)])
def test_documents(bad, code):
    big = 1 << 40
    refused(code, dh.dh_docs_plan, docs(**bad))
    refused(code, dh.dh_attn_docs_fwd, dh.DH_BF16, docs(**bad), 128, 0.0, A, A, A, A, big)
    refused(code, dh.dh_attn_docs_bwd, dh.DH_BF16, docs(**bad), 128, 0.0, A, A, A, A, A, A, A, big)


def test_attention():
    d, big = docs(), 1 << 40

    def both(code, dtype=dh.DH_BF16, dim=128, cap=0.0):
        refused(code, dh.dh_attn_docs_fwd, dtype, d, dim, cap, A, A, A, A, big)
        refused(code, dh.dh_attn_docs_bwd, dtype, d, dim, cap, A, A, A, A, A, A, A, big)

    both(dh.DH_ERR_INVALID_ARG, dtype=7)
    for dim in (32, 96, 256, 0, -64):
        both(dh.DH_ERR_SHAPE, dim=dim)
    for dim in (4, 264, 0):
        both(dh.DH_ERR_SHAPE, dtype=dh.DH_F32, dim=dim)
    for cap in (-1.0, float("nan"), float("inf"), 1e-4, 1001.0):
        both(dh.DH_ERR_INVALID_ARG, cap=cap)
    for i in range(3):
        for bad in (None, A + 8):
            p = [A, A, A]
            p[i] = bad
            if i < 2 or bad is None:
                refused(dh.DH_ERR_INVALID_ARG, dh.dh_attn_docs_fwd, dh.DH_BF16, d, 128, 0.0, *p, A, big)
    for i in range(6):
        for bad in (None, A + 8):
            p = [A] * 6
            p[i] = bad
            if i not in (3, 5) or bad is None:
                refused(dh.DH_ERR_INVALID_ARG, dh.dh_attn_docs_bwd, dh.DH_BF16, d, 128, 0.0, *p, A, big)
    for fn, n, size in ((dh.dh_attn_docs_fwd, 3, dh.dh_attn_docs_fwd_workspace_bytes), (dh.dh_attn_docs_bwd, 6, dh.dh_attn_docs_bwd_workspace_bytes)):
        need = size(dh.DH_BF16, 100, 4, 2, 128)
        if need:
            refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, fn, dh.DH_BF16, d, 128, 0.0, *[A] * n, A, need - 1)
            refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, fn, dh.DH_BF16, d, 128, 0.0, *[A] * n, None, need)
    with pytest.raises(dh.DhelixError):
        dh._check(dh.lib.dh_docs_plan(None, None))


def test_nothing_to_do_is_no_error():
    dh.dh_docs_plan(docs(T=0, table=None, doc_start=None))
    dh.dh_attn_docs_fwd(dh.DH_F32, docs(T=0), 64, 0.0, None, None, None)
    dh.dh_attn_docs_bwd(dh.DH_F32, docs(n_docs=0), 64, 0.0, None, None, None, None, None, None)
    dh.dh_rope_axes(dh.DH_F32, 0, 0, 0, (32,), None, 1, 64, 1e4, False, None, 64, None, 64)
    dh.dh_moe_balance_bwd(0, 4, None, None, None, None, None, False, None)
    assert dh.dh_docs_table_bytes(0, 1, 1) == 0 and dh.dh_moe_balance_ws_bytes(10, 1) == 0 and dh.dh_moe_balance_ws_bytes(10, 257) == 0
    assert dh.dh_attn_docs_fwd_workspace_bytes(dh.DH_BF16, 0, 4, 2, 128) == 0


def test_rope_axes():
    ok = dict(dtype=dh.DH_BF16, pairing=0, form=0, T=10, axis_pairs=(20, 44), pos=A, n_heads=2, head_dim=128, base=1e4, inverse=False, t=A, t_stride=256, out=A + 65536, out_stride=256)
    for bad, code in [(dict(dtype=5), dh.DH_ERR_INVALID_ARG), (dict(pairing=2), dh.DH_ERR_INVALID_ARG), (dict(form=-1), dh.DH_ERR_INVALID_ARG), (dict(base=0.0), dh.DH_ERR_INVALID_ARG),
                      (dict(base=float("nan")), dh.DH_ERR_INVALID_ARG), (dict(T=-1), dh.DH_ERR_SHAPE), (dict(n_heads=0), dh.DH_ERR_SHAPE), (dict(head_dim=120), dh.DH_ERR_SHAPE),
                      (dict(head_dim=528, t_stride=2048, out_stride=2048), dh.DH_ERR_SHAPE), (dict(t_stride=248), dh.DH_ERR_SHAPE), (dict(out_stride=260), dh.DH_ERR_SHAPE),
                      (dict(axis_pairs=()), dh.DH_ERR_SHAPE), (dict(axis_pairs=(10, 10, 10, 10, 24)), dh.DH_ERR_SHAPE), (dict(axis_pairs=(20, 43)), dh.DH_ERR_SHAPE),
                      (dict(axis_pairs=(20, 45)), dh.DH_ERR_SHAPE), (dict(axis_pairs=(0, 64)), dh.DH_ERR_SHAPE), (dict(axis_pairs=(-2 ** 31, 64)), dh.DH_ERR_SHAPE),
                      (dict(axis_pairs=(2 ** 31 - 1, 64)), dh.DH_ERR_SHAPE), (dict(pos=None), dh.DH_ERR_INVALID_ARG), (dict(t=None), dh.DH_ERR_INVALID_ARG),
                      (dict(out=None), dh.DH_ERR_INVALID_ARG), (dict(t=A + 8), dh.DH_ERR_INVALID_ARG), (dict(out=A + 4), dh.DH_ERR_INVALID_ARG),
                      (dict(out=A, out_stride=264), dh.DH_ERR_INVALID_ARG)]:
        refused(code, dh.dh_rope_axes, **{**ok, **bad})


def test_balance():
    need = dh.dh_moe_balance_ws_bytes(100, 16)
    ok = dict(T=100, E=16, logits=A, idx=A, n_live=None, counts=A, prob_mean=A, lse=A, loss=A, ws=A, ws_bytes=need)
    for bad, code in [(dict(T=-1), dh.DH_ERR_SHAPE), (dict(E=1), dh.DH_ERR_SHAPE), (dict(E=257), dh.DH_ERR_SHAPE), (dict(ws=None), dh.DH_ERR_WORKSPACE_TOO_SMALL),
                      (dict(ws_bytes=need - 1), dh.DH_ERR_WORKSPACE_TOO_SMALL),
                      (dict(ws=A + 2), dh.DH_ERR_INVALID_ARG)] + [({k: None}, dh.DH_ERR_INVALID_ARG) for k in ("logits", "idx", "counts", "prob_mean", "lse", "loss")]:
        refused(code, dh.dh_moe_balance_fwd, **{**ok, **bad})
    ok = dict(T=100, E=16, logits=A, lse=A, counts=A, n_live=None, dloss=A, accumulate=False, dlogits=A)
    for bad, code in [(dict(T=-1), dh.DH_ERR_SHAPE), (dict(E=1), dh.DH_ERR_SHAPE), (dict(E=300), dh.DH_ERR_SHAPE)] + [({k: None}, dh.DH_ERR_INVALID_ARG) for k in ("logits", "lse", "counts", "dloss", "dlogits")]:
        refused(code, dh.dh_moe_balance_bwd, **{**ok, **bad})


def tensors(**kw):
    f = dict(data=A, out=None, n=100, dtype=dh.DH_F32)
    f.update(kw)
    return (dh.dh_tensor * 1)(dh.dh_tensor(**f))


def test_gradients():
    for bad, code in [(dict(data=None), dh.DH_ERR_INVALID_ARG), (dict(data=A + 2), dh.DH_ERR_INVALID_ARG), (dict(out=A + 1, dtype=dh.DH_BF16), dh.DH_ERR_INVALID_ARG), (dict(dtype=9), dh.DH_ERR_INVALID_ARG),
                      (dict(n=1 << 47), dh.DH_ERR_SHAPE)]:
        refused(code, dh.dh_grad_norm, tensors(**bad), A, A, 1 << 40)
        refused(code, dh.dh_grad_clip, tensors(**bad), A, 1.0)
    t = tensors()
    need = dh.dh_grad_norm_ws_bytes(t)
    assert need > 0 and dh.dh_grad_norm_ws_bytes((dh.dh_tensor * 0)()) == 0
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_grad_norm, t, A, A, need - 1)
    refused(dh.DH_ERR_WORKSPACE_TOO_SMALL, dh.dh_grad_norm, t, A, None, need)
    refused(dh.DH_ERR_INVALID_ARG, dh.dh_grad_norm, t, A, A + 4, need)
    refused(dh.DH_ERR_INVALID_ARG, dh.dh_grad_norm, t, None, A, need)
    refused(dh.DH_ERR_INVALID_ARG, dh.dh_grad_clip, t, None, 1.0)
    for m in (0.0, -1.0, float("nan")):
        refused(dh.DH_ERR_INVALID_ARG, dh.dh_grad_clip, t, A, m)
    with pytest.raises(dh.DhelixError):
        dh._check(dh.lib.dh_grad_clip(-1, t, A, 1.0, None))
    with pytest.raises(dh.DhelixError):
        dh._check(dh.lib.dh_grad_norm(2, C.POINTER(dh.dh_tensor)(), A, A, 100, None))
    import torch
    with pytest.raises(ValueError):
        dh.tensor_list([torch.zeros(4, dtype=torch.float16)])
    with pytest.raises(ValueError):
        dh.tensor_list([torch.zeros((4, 4)).t()])
    with pytest.raises(ValueError):
        dh.tensor_list([torch.zeros(4)], [torch.zeros(5)])


@pytest.mark.parametrize("T,nq,nkv", [(1 << 28, 1024, 1), (1 << 28, 512, 1), (1 << 27, 1024, 1), (1 << 28, 1000, 2)])
def test_more_tiles_of_a_group_than_are_counted(T, nq, nkv):
    """A key block of one document meets T/64 tiles of each head of its group, and the work lists count these in 32 bits."""
    assert T // 64 * (nq // nkv) > 1 << 30
    bad = dict(T=T, nq=nq, nkv=nkv)
    refused(dh.DH_ERR_SHAPE, dh.dh_docs_plan, docs(**bad))
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_fwd, dh.DH_BF16, docs(**bad), 128, 0.0, A, A, A, A, 1 << 60)
    refused(dh.DH_ERR_SHAPE, dh.dh_attn_docs_bwd, dh.DH_BF16, docs(**bad), 128, 0.0, A, A, A, A, A, A, A, 1 << 60)


@pytest.mark.parametrize("parts", [[(0, None, 100), (0, None, 100)],                   # a tensor twice, in place
                                   [(0, None, 100), (396, None, 100)],                 # one element shared
                                   [(0, 400, 100), (1000, 400, 100)],                  # two results in one place
                                   [(0, 1200, 100), (1000, 2000, 100)],                # a result over another tensor
                                   [(0, 4, 100)],                                      # a result shifted over its own tensor
                                   [(0, 40000, 10000), (80000, None, 10), (80036, None, 10), (90000, None, 5)]])
def test_clipping_what_overlaps(parts):
    t = (dh.dh_tensor * len(parts))(*[dh.dh_tensor(A + d, None if o is None else A + o, n, dh.DH_F32) for d, o, n in parts])
    refused(dh.DH_ERR_INVALID_ARG, dh.dh_grad_clip, t, A, 1.0)
