"""Host-side checks of the routed experts in training and of the norms: bad arguments are refused before anything
is enqueued.  CPU only."""
import ctypes

import pytest
import torch

import paper_2608_16157_amd as ftm

F = 0x10000        # a device address that is never used: every call here is refused or has no tokens
ref = ctypes.byref
OK, NULL, SHAPE, DTYPE, CAPACITY = ftm.FT_OK, ftm.FT_ERR_NULL, ftm.FT_ERR_SHAPE, ftm.FT_ERR_DTYPE, ftm.FT_ERR_CAPACITY
BAD_DESCS = [dict(n_experts=0), dict(n_experts=1025), dict(top_k=0), dict(top_k=9), dict(n_experts=128, top_k=65),
             dict(first=-1), dict(local=0), dict(first=1), dict(local=9), dict(align=64), dict(align=0), dict(rows=0),
             dict(rows=100), dict(rows=1 << 21), dict(align=128, rows=144)]


def desc(**kw):
    return {"n_experts": 8, "top_k": 2, "first": 0, "local": 8, "align": 16, "rows": 128, **kw}


def dref(d):
    return ref(ftm.ft_sort_desc_t(*[d[n] for n, _ in ftm.ft_sort_desc_t._fields_]))


def tables(**kw):
    return ref(ftm.ft_sort_t(**{**dict.fromkeys(("row_pair", "pair_row", "off", "count", "dropped"), F), **kw}))


def codes(c=F, s=F):
    return ref(ftm.ft_act_codes_t(c, s))


def sort(d=desc(), ids=F, T=4, mask=None, out=tables(), ws=F, n=1 << 30):
    return ftm.load().ft_expert_sort(dref(d), ids, T, mask, out, ws, n, None)


def gather(d=desc(), s=tables(), x=F, xd=1, T=4, C=128, w=None, plain=F, pd=1, row=None, col=None):
    return ftm.load().ft_expert_gather(dref(d), s, x, xd, T, C, w, plain, pd, row, col, None)


def combine(d=desc(), s=tables(), rows=F, rd=1, T=4, C=128, w=None, base=None, y=F, yd=1):
    return ftm.load().ft_expert_combine(dref(d), s, rows, rd, T, C, w, base, y, yd, None)


def gate_grad(d=desc(), s=tables(), rows=F, rd=1, dy=F, yd=1, T=4, C=128, dw=F):
    return ftm.load().ft_expert_gate_grad(dref(d), s, rows, rd, dy, yd, T, C, dw, None)


def linear(d=desc(), out=128, inn=256, xd=4, yd=1, w=F, ws=F, x=codes(), s=tables(), T=4, y=F):
    return ftm.load().ft_expert_linear(dref(d), ref(ftm.ft_linear_desc_t(out, inn, xd, yd)), w, ws, x, s, T, y, None)


def weight_grad(d=desc(align=128), N=128, K=256, dy=codes(), x=codes(), s=tables(), T=4, dw=F, dt=0, acc=0):
    return ftm.load().ft_expert_weight_grad(dref(d), N, K, dy, x, s, T, dw, dt, acc, None)


@pytest.mark.parametrize("bad", BAD_DESCS)
def test_bad_layouts_are_refused(bad):
    d = desc(**bad)
    for call in (sort, gather, combine, gate_grad, linear):
        assert call(d=d) == SHAPE, call.__name__
    assert weight_grad(d={**d, "align": bad.get("align", 128)}) == SHAPE
    assert ftm.ft_expert_sort_workspace_bytes(d, 4) == 0
    assert sort(d=desc(), T=-1) == sort(d=desc(), T=(1 << 20) + 1) == SHAPE


def test_sort_refuses():
    assert sort(ids=None) == sort(out=None) == sort(ws=None) == NULL
    assert ftm.load().ft_expert_sort(None, F, 4, None, tables(), F, 1 << 30, None) == NULL
    for n in ("row_pair", "pair_row", "off", "count", "dropped"):
        assert sort(out=tables(**{n: None})) == NULL
        assert sort(out=tables(**{n: F + 2})) == SHAPE
    assert sort(n=16) == CAPACITY
    assert sort(ws=F + 8) == sort(ids=F + 1) == SHAPE


def test_sort_sizes():
    rows = lambda T, **kw: ftm.ft_expert_sort_rows(desc(**kw), T)
    assert rows(0) == 16 and rows(0, align=128) == 128
    assert rows(1) == 32 and rows(1, align=128) == 256          # two pairs, two groups of one
    assert rows(4) == 128 and rows(100) == 320                  # 200 pairs, 8 groups: 200 + 8 * 15 = 320
    assert rows(1 << 20) == 0 and rows(-1) == 0 and rows(4, first=1) == 0
    assert rows(520000) == 1040112 and ftm.ft_expert_sort_rows({"n_experts": 8, "top_k": 2, "align": 16}, 4) == 128
    sizes = [ftm.ft_expert_sort_workspace_bytes(desc(rows=1 << 20), T) for T in (0, 1, 2048, 2049, 100000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    with pytest.raises(ftm.FtError):
        ftm.alloc_sort_workspace(desc(align=3), 4, device="cpu")


def test_rows_calls_refuse():
    assert gather(C=8) == gather(C=100) == gather(C=65552) == gather(T=-1) == gather(x=F + 8) == gather(plain=F + 4) == SHAPE
    assert gather(w=F + 2) == gather(row=codes(F + 4)) == gather(s=tables(off=F + 1)) == SHAPE
    assert gather(plain=None, col=codes()) == SHAPE              # column forms need groups of whole blocks
    assert gather(xd=2) == gather(pd=4) == DTYPE
    assert gather(x=None) == gather(plain=None) == gather(row=codes(None)) == gather(s=None) == NULL
    assert gather(s=tables(row_pair=None)) == gather(s=tables(off=None)) == NULL
    assert combine(C=24) == combine(T=1 << 21) == combine(rows=F + 8) == combine(y=F + 2) == combine(base=F + 8) == SHAPE
    assert combine(w=F + 1) == combine(s=tables(pair_row=F + 1)) == SHAPE
    assert combine(rd=2) == combine(yd=4) == DTYPE
    assert combine(rows=None) == combine(y=None) == combine(s=None) == combine(s=tables(pair_row=None)) == NULL
    assert gate_grad(C=0) == gate_grad(rows=F + 1) == gate_grad(dy=F + 8) == gate_grad(dw=F + 2) == SHAPE
    assert gate_grad(rd=4) == gate_grad(yd=3) == DTYPE
    assert gate_grad(rows=None) == gate_grad(dy=None) == gate_grad(dw=None) == gate_grad(s=tables(pair_row=None)) == NULL
    assert gather(T=0, x=None) == combine(T=0, rows=None) == gate_grad(T=0, dy=None) == OK


def test_products_refuse():
    assert linear(out=24) == linear(inn=0) == linear(T=-1) == linear(w=F + 1) == linear(y=F + 8) == linear(ws=F + 2) == SHAPE
    assert linear(x=codes(F + 1)) == linear(s=tables(count=F + 1)) == SHAPE
    assert linear(xd=1) == linear(yd=2) == DTYPE
    assert linear(w=None) == linear(ws=None) == linear(y=None) == linear(x=None) == linear(x=codes(F, None)) == linear(s=None) == NULL
    assert linear(s=tables(off=None)) == linear(s=tables(count=None)) == NULL
    assert linear(T=0, w=None) == OK
    assert ftm.load().ft_expert_linear(dref(desc()), None, F, F, codes(), tables(), 4, F, None) == NULL
    tr = lambda n=3, N=128, K=128, w=F, s=F, wt=F, st=F: ftm.load().ft_expert_linear_transpose(n, N, K, w, s, wt, st, None)
    assert tr(n=0) == tr(n=1025) == tr(N=8) == tr(K=130) == tr(w=F + 1) == tr(wt=F + 8) == tr(st=F + 1) == SHAPE
    assert tr(w=None) == tr(s=None) == tr(wt=None) == tr(st=None) == NULL
    assert weight_grad(d=desc()) == weight_grad(N=8) == weight_grad(K=100) == weight_grad(acc=2) == weight_grad(dw=F + 4) == SHAPE
    assert weight_grad(dy=codes(F + 1)) == weight_grad(s=tables(off=F + 2)) == SHAPE
    assert weight_grad(dt=2) == weight_grad(dt=1, acc=1) == DTYPE
    assert weight_grad(dw=None) == weight_grad(dy=None) == weight_grad(x=None) == weight_grad(s=None) == NULL
    assert weight_grad(s=tables(count=None)) == NULL
    assert weight_grad(T=0, acc=1, dy=None, s=None) == OK


def norm(C=128, xd=1, yd=1, wd=0, post=1, eps=1e-6, scale=1.0, params=None, x=F, b=F, T=4, r=F, n=F, row=None):
    d = ftm.ft_norm_desc_t(C, xd, yd, wd, post, eps, scale)
    return ftm.load().ft_block_norm(ref(d), ref(params or ftm.ft_norm_params_t(F, F, F, F)), x, b, T, r, n, row, None)


def back(C=128, xd=1, yd=1, wd=0, post=1, eps=1e-6, scale=1.0, params=None, r=F, b=F, dr=F, dn=F, T=4, dx=F, db=F,
         grads=(F, F, F, F), ws=F, n=1 << 30):
    d, g = ftm.ft_norm_desc_t(C, xd, yd, wd, post, eps, scale), None if grads is None else ref(ftm.ft_norm_grads_t(*grads))
    return ftm.load().ft_block_norm_backward(ref(d), ref(params or ftm.ft_norm_params_t(F, F, F, F)), r, b, dr, dn, T, dx, db,
                                             g, ws, n, None)


def test_norms_refuse():
    bad = ftm.ft_norm_params_t
    for call in (norm, back):
        assert call(C=8) == call(C=65552) == call(post=2) == call(eps=-1.0) == call(eps=float("nan")) == call(T=-1) == SHAPE
        assert call(scale=float("inf")) == call(eps=float("inf")) == call(T=1 << 21) == SHAPE
        assert call(xd=2) == call(yd=4) == call(wd=3) == DTYPE
        assert call(params=bad(F + 4, F, F, F)) == call(params=bad(F, F, F + 8, F)) == call(params=bad(F, F, F, F + 2)) == SHAPE
    lib, d = ftm.load(), ftm.ft_norm_desc_t(128, 1, 1, 1, 0, 0.0, 1.0)
    assert lib.ft_block_norm(ref(d), None, F, F, 4, F, F, None, None) == NULL
    assert lib.ft_block_norm(None, ref(bad()), F, F, 4, F, F, None, None) == NULL
    assert norm(x=None) == norm(r=None, n=None) == norm(b=None, n=None) == norm(row=codes(F, None)) == NULL
    assert norm(x=F + 2) == norm(b=F + 8) == norm(r=F + 8) == norm(n=F + 4) == norm(row=codes(F + 1)) == SHAPE
    assert norm(T=0, x=None) == OK
    assert back(r=None) == back(dr=None, dn=None) == back(dn=None) == back(b=None) == NULL          # pre needs dn
    assert back(dx=None, db=None, grads=None) == back(post=0) == back(ws=None) == NULL
    assert back(b=None, db=None, grads=(F, None, F, None)) == back(b=None, db=None, grads=(F, None, None, F)) == NULL
    assert back(n=64) == CAPACITY
    assert back(r=F + 8) == back(dr=F + 2) == back(dx=F + 8) == back(ws=F + 4) == back(grads=(F + 1, F, F, F)) == SHAPE
    assert back(T=0, grads=None) == back(T=0, grads=(None, None, None, F), ws=None) == OK
    nd = {"channels": 7168, "x_dtype": 1, "y_dtype": 1, "w_dtype": 0, "post_norm": 1, "eps": 1e-6}
    sizes = [ftm.ft_block_norm_workspace_bytes(nd, T) for T in (0, 1, 100, 5000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] >= 2 * 7168 * 4
    assert ftm.ft_block_norm_workspace_bytes({**nd, "channels": 100}, 4) == 0
    with pytest.raises(ftm.FtError):
        ftm.alloc_block_norm_workspace({**nd, "w_dtype": 7}, 4, device="cpu")


def test_binding_refuses_before_the_call():
    d = desc()
    s = ftm.SortBuffers(d, 4, device="cpu")
    assert s.row_pair.shape == (128,) and s.pair_row.shape == (4, 2) and s.off.shape == (9,)
    x, w = torch.zeros(4, 128, dtype=torch.bfloat16), torch.zeros(4, 2)
    c = ftm.ActCodes(128, 128, device="cpu")
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    lin = {"out_features": 128, "in_features": 128, "x_dtype": ftm.FT_DT_FP8_ACT, "y_dtype": ftm.FT_DT_BF16}
    wt = {"w": torch.zeros(8, 128, 128, dtype=torch.uint8), "s": torch.ones(8, 1, 1)}
    nd = {"channels": 128, "x_dtype": ftm.FT_DT_BF16, "y_dtype": ftm.FT_DT_BF16, "w_dtype": ftm.FT_DT_F32, "eps": 1e-6}
    for call in (lambda: ftm.ft_expert_sort(d, torch.zeros(4, 2, dtype=torch.int32), 4, s, ws),
                 lambda: ftm.ft_expert_gather(d, s, x, 4, 128, row=c),
                 lambda: ftm.ft_expert_combine(d, s, torch.zeros(128, 128), 4, 128, x),
                 lambda: ftm.ft_expert_gate_grad(d, s, torch.zeros(128, 128), x, 4, 128, w),
                 lambda: ftm.ft_expert_linear(d, lin, wt, c, s, 4, torch.zeros(128, 128, dtype=torch.bfloat16)),
                 lambda: ftm.ft_expert_weight_grad(d, 128, 128, c, c, s, 4, torch.zeros(8, 128, 128)),
                 lambda: ftm.ft_block_norm(nd, {}, x, None, 4, n=x),
                 lambda: ftm.ft_block_norm_backward(nd, {}, x, None, None, x, 4, dx=x)):
        with pytest.raises(ValueError, match="device"):
            call()
    with pytest.raises(ValueError, match="SortBuffers"):
        ftm._groups_arg(-1, ftm._sort_desc(d), None)
    for call in (lambda: ftm.ft_expert_gather(d, s, x, 4, 100, row=c), lambda: ftm.ft_expert_combine(d, s, x, -1, 128, x),
                 lambda: ftm.ft_expert_linear_transpose(0, 128, 128, wt, wt), lambda: ftm.ft_block_norm({**nd, "x_dtype": 4}, {}, x, None, 4),
                 lambda: ftm.ft_expert_linear(d, {**lin, "x_dtype": 1}, wt, c, s, 4, x),
                 lambda: ftm.ft_block_norm({**nd, "channels": 24}, {}, x, None, 4)):
        with pytest.raises(ftm.FtError):
            call()
    # calls without tokens reach neither the library nor a device
    ftm.ft_expert_gather(d, s, x, 0, 128, row=c)
    ftm.ft_expert_combine(d, s, x, 0, 128, x)
    ftm.ft_expert_gate_grad(d, s, x, x, 0, 128, w)
    ftm.ft_expert_linear(d, lin, {}, c, s, 0, x)
    ftm.ft_block_norm(nd, {}, x, None, 0)
    ftm.ft_block_norm_backward(nd, {}, x, None, None, x, 0, dx=x)
