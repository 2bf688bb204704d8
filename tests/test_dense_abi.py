"""Host-side checks of the dense 8-bit operators and the balance loss: bad arguments are refused before
anything is enqueued.  CPU only."""
import ctypes

import pytest
import torch

import paper_2608_16157_amd as ftm

F = 0x10000        # a device address that is never used: every call here is refused or has no tokens
ref = ctypes.byref


def codes(c=F, s=F):
    return ftm.ft_act_codes_t(c, s)


def test_act_quantize_refuses():
    lib, c = ftm.load(), codes()
    call = lambda x=F, dt=1, T=4, C=128, row=ref(c), col=None: lib.ft_act_quantize(x, dt, T, C, row, col, None)
    assert call(C=8) == call(C=100) == call(C=65552) == call(T=-1) == call(T=1 << 21) == ftm.FT_ERR_SHAPE
    assert call(dt=2) == call(dt=4) == ftm.FT_ERR_DTYPE
    assert call(x=None) == call(row=None) == call(row=ref(codes(None))) == call(col=ref(codes(F, None))) == ftm.FT_ERR_NULL
    assert call(x=F + 8) == call(row=ref(codes(F + 4))) == call(col=ref(codes(F, F + 1))) == ftm.FT_ERR_SHAPE
    assert call(T=0) == call(T=0, x=None) == ftm.FT_OK


def linear(out=128, inn=256, xd=1, yd=1, w=F, s=F, x=F, xs=None, T=4, y=F, ws=F, n=1 << 30):
    d = ftm.ft_linear_desc_t(out, inn, xd, yd)
    return ftm.load().ft_linear(ref(d), w, s, x, xs, T, y, ws, n, None)


@pytest.mark.parametrize("kw,want", [
    (dict(out=24), ftm.FT_ERR_SHAPE), (dict(inn=0), ftm.FT_ERR_SHAPE), (dict(out=65552), ftm.FT_ERR_SHAPE),
    (dict(T=-1), ftm.FT_ERR_SHAPE), (dict(T=(1 << 20) + 1), ftm.FT_ERR_SHAPE),
    (dict(xd=2), ftm.FT_ERR_DTYPE), (dict(yd=2), ftm.FT_ERR_DTYPE), (dict(yd=4), ftm.FT_ERR_DTYPE),
    (dict(w=None), ftm.FT_ERR_NULL), (dict(s=None), ftm.FT_ERR_NULL), (dict(x=None), ftm.FT_ERR_NULL),
    (dict(y=None), ftm.FT_ERR_NULL), (dict(ws=None), ftm.FT_ERR_NULL), (dict(xd=4), ftm.FT_ERR_NULL),
    (dict(n=64), ftm.FT_ERR_CAPACITY), (dict(xd=4, xs=F, n=64), ftm.FT_ERR_CAPACITY), (dict(w=F + 1), ftm.FT_ERR_SHAPE), (dict(x=F + 8), ftm.FT_ERR_SHAPE),
    (dict(y=F + 2), ftm.FT_ERR_SHAPE), (dict(ws=F + 4), ftm.FT_ERR_SHAPE), (dict(s=F + 2), ftm.FT_ERR_SHAPE),
    (dict(xd=4, xs=F + 3), ftm.FT_ERR_SHAPE), (dict(T=0), ftm.FT_OK), (dict(T=0, x=None, ws=None), ftm.FT_OK),
])
def test_linear_refuses(kw, want):
    assert linear(**kw) == want
    assert ftm.load().ft_linear(None, F, F, F, None, 4, F, F, 1 << 30, None) == ftm.FT_ERR_NULL


def test_linear_workspace():
    d = {"out_features": 48, "in_features": 144, "x_dtype": ftm.FT_DT_BF16, "y_dtype": ftm.FT_DT_BF16}
    sizes = [ftm.ft_linear_workspace_bytes(d, T) for T in (0, 1, 16, 17, 128, 129, 5000)]
    assert sizes == sorted(sizes) and sizes[0] >= 256 * 128 + 256
    assert sizes[-1] >= 5120 * 256 + 5120 * 2
    assert 0 < ftm.ft_linear_workspace_bytes(dict(d, x_dtype=ftm.FT_DT_FP8_ACT), 100) < ftm.ft_linear_workspace_bytes(d, 100)
    assert ftm.ft_linear_workspace_bytes(dict(d, in_features=100), 100) == 0
    with pytest.raises(ftm.FtError):
        ftm.alloc_linear_workspace(dict(d, y_dtype=9), 100, device="cpu")


def test_transpose_and_weight_grad_refuse():
    lib, c = ftm.load(), codes()
    tr = lambda n=128, k=128, w=F, s=F, wt=F, st=F: lib.ft_linear_transpose(n, k, w, s, wt, st, None)
    assert tr(n=8) == tr(k=130) == tr(w=F + 1) == tr(wt=F + 8) == tr(st=F + 1) == ftm.FT_ERR_SHAPE
    assert tr(w=None) == tr(s=None) == tr(wt=None) == tr(st=None) == ftm.FT_ERR_NULL
    wg = lambda n=128, k=128, T=8, dy=ref(c), x=ref(c), dw=F, dt=0, acc=0: lib.ft_linear_weight_grad(n, k, T, dy, x, dw, dt, acc, None)
    assert wg(n=8) == wg(k=65600) == wg(T=-1) == wg(acc=2) == wg(dw=F + 4) == wg(dy=ref(codes(F + 1))) == ftm.FT_ERR_SHAPE
    assert wg(dt=2) == wg(dt=1, acc=1) == ftm.FT_ERR_DTYPE
    assert wg(dw=None) == wg(dy=None) == wg(x=None) == wg(x=ref(codes(F, None))) == ftm.FT_ERR_NULL
    assert wg(T=0, acc=1, dy=None) == ftm.FT_OK


def test_swiglu_refuses():
    lib, c = ftm.load(), codes()
    fw = lambda gu=F, dt=1, T=4, I=128, h=ref(c), sv=ref(c): lib.ft_swiglu_quantize(gu, dt, T, I, h, sv, None)
    assert fw(I=64) == fw(I=192) == fw(I=32896) == fw(T=-1) == fw(gu=F + 2) == fw(h=ref(codes(F, F + 8))) == ftm.FT_ERR_SHAPE
    assert fw(dt=4) == ftm.FT_ERR_DTYPE
    assert fw(gu=None) == fw(h=None) == fw(sv=ref(codes(None, F))) == ftm.FT_ERR_NULL
    assert fw(T=0, gu=None) == ftm.FT_OK
    bw = lambda sv=ref(c), dh=F, dt=1, T=4, I=128, a=ref(c), b=None, h=None: lib.ft_swiglu_backward(sv, dh, dt, T, I, a, b, h, None)
    assert bw(I=100) == bw(T=1 << 21) == bw(dh=F + 8) == bw(b=ref(codes(F + 1))) == ftm.FT_ERR_SHAPE
    assert bw(dt=3) == ftm.FT_ERR_DTYPE
    assert bw(sv=None) == bw(dh=None) == bw(a=None) == bw(h=ref(codes(None))) == ftm.FT_ERR_NULL
    assert bw(T=0, dh=None) == ftm.FT_OK


def test_balance_refuses():
    lib = ftm.load()
    out = ftm.ft_balance_t(F, F, F, F, F)

    def call(E=8, k=2, gating=0, n=1, logits=F, ids=F, T=4, off=None, o=ref(out), ws=F, nb=1 << 30):
        d = ftm.ft_balance_desc_t(E, k, gating, n, 1.0)
        return lib.ft_balance_loss(ref(d), logits, ids, T, off, None, o, ws, nb, None)

    assert call(E=0) == call(E=1025) == call(k=9) == call(k=0) == call(n=0) == call(n=65537) == call(T=-1) == ftm.FT_ERR_SHAPE
    assert call(E=128, k=65) == call(ws=F + 8) == ftm.FT_ERR_SHAPE
    assert call(gating=2) == ftm.FT_ERR_DTYPE
    assert call(logits=None) == call(ids=None) == call(n=2) == call(o=None) == call(ws=None) == ftm.FT_ERR_NULL
    assert call(o=ref(ftm.ft_balance_t(F, F, F, None, F))) == ftm.FT_ERR_NULL
    assert call(nb=16) == ftm.FT_ERR_CAPACITY

    def back(E=8, k=2, gating=0, n=1, logits=F, ids=F, T=4, off=None, b=ref(out), dl=F, w=F, dw=F, d=F):
        desc = ftm.ft_balance_desc_t(E, k, gating, n, 1.0)
        return lib.ft_router_backward(ref(desc), logits, ids, T, off, None, b, dl, w, dw, d, None)

    assert back(E=2000) == back(T=1 << 21) == ftm.FT_ERR_SHAPE
    assert back(gating=5) == ftm.FT_ERR_DTYPE
    assert back(logits=None) == back(d=None) == back(dl=None, dw=None) == back(n=3) == ftm.FT_ERR_NULL
    assert back(b=None) == back(b=ref(ftm.ft_balance_t(F, None, F, F, F))) == back(w=None) == back(ids=None) == ftm.FT_ERR_NULL
    assert back(T=0, logits=None) == ftm.FT_OK
    d = {"n_experts": 256, "top_k": 8, "gating": 1, "n_seq": 9}
    sizes = [ftm.ft_balance_workspace_bytes(d, T) for T in (0, 1, 512, 513, 8192, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert ftm.ft_balance_workspace_bytes(dict(d, n_seq=0), 4) == 0


def test_binding_refuses_before_the_call():
    x = torch.zeros(4, 128, dtype=torch.bfloat16)
    c = ftm.ActCodes(4, 128, device="cpu")
    with pytest.raises(ValueError, match="device"):
        ftm.ft_act_quantize(x, 4, 128, c)
    with pytest.raises(ftm.FtError):
        ftm.ft_act_quantize(x, 4, 100, c)
    assert c.codes.shape == (4, 128) and c.scales.shape == (1, 128)
    assert ftm.ActCodes(130, 144, device="cpu").scales.shape == (2, 256)
    d = {"out_features": 128, "in_features": 128, "x_dtype": ftm.FT_DT_FP8_ACT, "y_dtype": ftm.FT_DT_BF16}
    with pytest.raises(ValueError, match="device"):
        ftm.ft_linear(d, {"w": torch.zeros(128, 128, dtype=torch.uint8), "s": torch.ones(1, 1)}, c, 4, x)
    with pytest.raises(ValueError, match="4 x 128"):
        ftm._need_codes(c, "x", 5, 128)
    with pytest.raises(ftm.FtError):
        ftm.ft_linear_transpose(100, 128, {}, {})
    with pytest.raises(ValueError, match="expected a torch.Tensor"):
        ftm.ft_linear_weight_grad(128, 128, 4, c, c, None)
    with pytest.raises(ftm.FtError):
        ftm.ft_swiglu_quantize(x, 4, 64, c)
    with pytest.raises(ValueError, match="device"):
        ftm.ft_swiglu_backward(ftm.ActCodes(4, 256, device="cpu"), x, 4, 128, c)
    bd = {"n_experts": 8, "top_k": 2, "gating": 0, "n_seq": 1}
    with pytest.raises(ValueError, match="device"):
        ftm.ft_balance_loss(bd, torch.zeros(4, 8), torch.zeros(4, 2, dtype=torch.int32), 4, None, None)
    with pytest.raises(ValueError, match="device"):
        ftm.ft_router_backward(bd, torch.zeros(4, 8), None, 4, None, None, None)
    # calls without tokens reach neither the library nor a device
    ftm.ft_act_quantize(x, 0, 128, c)
    ftm.ft_linear(d, {}, c, 0, x)
    ftm.ft_swiglu_quantize(x, 0, 128, c)
    ftm.ft_swiglu_backward(c, x, 0, 128, c)
