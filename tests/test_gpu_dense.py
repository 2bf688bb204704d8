"""The dense 8-bit operators and the router's balance loss on the GPU against the 64-bit oracle.

Tolerances, from the arithmetic:
* 8-bit forms of given data are exact (codes and scales equal the oracle's);
* 8-bit forms of computed values: half a step of e4m3fn (2^-4 of the value, 2^-10 of the scale among the
  subnormal codes) beyond the float32 value, whose own error is below 2^-16 of it; a scale may differ
  only where the block's largest magnitude lies that near a border;
* float32 products: codes and scaled codes are exact, so at most K roundings of the sums and one per block
  of its scale, (K + K/128 + 2) 2^-24 sum|ab|;
* bf16 products: one rounding (2^-8 of the value) beyond the fp8 matrix instructions' sum, for whose error
  2^-11 sum|ab| of a block is allowed (the largest of many measured blocks: 2.9e-4);
* router probabilities: arguments of exp up to 100 round to 100 * 2^-24, and some ten further roundings;
  sums over n tokens n 2^-24: below 2e-5 of the sum of magnitudes for the sizes here.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_16157_amd as ftm
from oracle import dense

pytestmark = pytest.mark.gpu
BF16, F32, ACT = ftm.FT_DT_BF16, ftm.FT_DT_F32, ftm.FT_DT_FP8_ACT
TORCH = {BF16: torch.bfloat16, F32: torch.float32}


def rng(*key):
    return np.random.default_rng(list(key))


def cuda(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().double().cpu().numpy()


def matrix(r, R, K, dtype=BF16, spread=3):
    """Values of many magnitudes, as float64 of what the tensor holds, and the tensor."""
    x = r.normal(size=(R, K)) * 10.0 ** r.uniform(-spread, spread, (R, 1))
    x[r.random((R, K)) < 0.02] = 0.0
    t = cuda(x).to(TORCH[dtype])
    return f64(t), t


def filled(R, K):
    """A form whose buffers hold other bytes than the call should leave."""
    c = ftm.ActCodes(R, K)
    c.codes.fill_(0xA5)
    c.scales.fill_(0x5A)
    return c


def form_of(x):
    """The 8-bit form of x [R][K] from the oracle, on the GPU."""
    codes, s = dense.quantize(x)
    full = np.full((s.shape[0], dense.pad128(x.shape[0])), 127, np.uint8)
    full[:, :x.shape[0]] = s
    return ftm.ActCodes.of(cuda(codes), cuda(full), *x.shape), dense.values(codes, s)[:, :x.shape[1]]


def weight(r, N, K):
    Np, Kp = dense.pad128(N), dense.pad128(K)
    w = r.integers(0, 256, (N, Kp)).astype(np.uint8)
    w[(w & 0x7F) == 0x7F] = 0x3A
    w[:, K:] = 0
    s = r.uniform(0.2, 2.0, (Np // 128, Kp // 128)).astype(np.float32) * 0.01
    s[r.random(s.shape) < 0.1] = 0.0
    return {"w": cuda(w), "s": cuda(s)}, dense.weight_values(w, s)[:, :K]


def assert_exact_form(c, x):
    codes, s = dense.quantize(x)
    R = x.shape[0]
    assert np.array_equal(c.codes.cpu().numpy(), codes)
    got = c.scales.cpu().numpy()
    assert np.array_equal(got[:, :R], s) and np.all(got[:, R:] == 127)


def assert_near_form(c, v):
    """c is the form of v up to v's float32 error."""
    R, K = v.shape
    got, s = c.codes.cpu().numpy(), c.scales.cpu().numpy()
    assert not got[:, K:].any() and np.all(s[:, R:] == 127)
    s = s[:, :R].astype(float)
    b = np.zeros((R, got.shape[1]))
    b[:, :K] = v
    amax = np.abs(b.reshape(R, -1, 128)).max(axis=2).T
    scale = 2.0 ** (s - 127)
    live = amax > 1e-37
    assert np.all(448 * scale[live] >= amax[live] * (1 - 2.0 ** -16))
    assert np.all(448 * scale[live] / 2 < amax[live] * (1 + 2.0 ** -16))
    err = np.abs(dense.values(got, s.astype(np.uint8)) - b)
    half = np.maximum(2.0 ** -4 * np.abs(b), 2.0 ** -10 * np.repeat(scale.T, 128, axis=1))
    assert np.all(err <= half * (1 + 2.0 ** -8) + 2.0 ** -16 * np.abs(b))


def assert_product(y, want, mag, K, dtype):
    """y against want = sum ab, mag = sum |ab| (K terms)."""
    tol = (K + K // 128 + 2) * 2.0 ** -24 * mag if dtype == F32 else 2.0 ** -8 * np.abs(want) + 2.0 ** -11 * mag
    err = np.abs(f64(y).reshape(want.shape) - want)
    assert np.all(err <= tol + 1e-37), float((err - tol).max())


TOKENS = (1, 2, 15, 16, 17, 48, 64, 65, 127, 128, 129, 300)
SHAPES = ((16, 16), (48, 144), (128, 128), (272, 384), (576, 1040), (2048, 256))   # (N, K)


# ------------------------------------------------------------------------------- 8-bit forms

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("T,C", ((1, 16), (1, 128), (3, 48), (127, 144), (128, 128), (129, 272), (300, 1040)))
def test_quantize_is_exact(T, C, dtype):
    x, t = matrix(rng(T, C), T, C, dtype, spread=8)
    row, col = filled(T, C), filled(C, T)
    ftm.ft_act_quantize(t, T, C, row, col)
    assert_exact_form(row, x)
    assert_exact_form(col, x.T)
    only = filled(T, C), filled(C, T)
    ftm.ft_act_quantize(t, T, C, row=only[0])
    ftm.ft_act_quantize(t, T, C, col=only[1])
    for a, b in zip(only, (row, col)):
        assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)


def test_quantize_of_extreme_values():
    """Blocks of zeros, of subnormals, at the borders of a scale, at the type's largest value, and values
    that are not finite: NaN codes, the rest of their block as if they were not there."""
    x = np.zeros((9, 256), np.float32)
    x[1, :128] = 1e-45
    x[2, 5] = 448.0
    x[3, 5] = np.nextafter(np.float32(448), np.float32(500))
    x[4] = np.linspace(-3.4e38, 3.4e38, 256)
    x[5, :] = 2.0 ** -120
    x[6, :4] = (np.inf, -np.inf, np.nan, 7.0)
    x[7, 200] = -np.inf
    x[8] = 2.0 ** np.linspace(-149, 0, 256)
    # a signalling NaN in an otherwise ordinary block
    x.view(np.uint32)[2, 130] = 0x7F800001
    x.view(np.uint32)[3, 131] = 0xFF810000
    row, col = filled(9, 256), filled(256, 9)
    ftm.ft_act_quantize(cuda(x), 9, 256, row, col)
    alone = filled(9, 256)
    ftm.ft_act_quantize(cuda(x), 9, 256, row=alone)
    assert torch.equal(alone.codes, row.codes) and torch.equal(alone.scales, row.scales)
    for c, v in ((row, x), (col, x.T)):
        codes, s = dense.quantize(v.astype(np.float64))
        got = c.codes.cpu().numpy()
        nan = (codes & 0x7F) == 0x7F
        assert nan.any() and np.array_equal((got & 0x7F) == 0x7F, nan)
        assert np.array_equal(got[~nan], codes[~nan])
        assert np.array_equal(c.scales.cpu().numpy()[:, :v.shape[0]], s)


# ------------------------------------------------------------------------------ dense product

def run_linear(N, K, T, wt, x, xd, yd, **kw):
    d = {"out_features": N, "in_features": K, "x_dtype": xd, "y_dtype": yd}
    y = torch.full((T + 1, N), 7.0, dtype=TORCH[yd], device="cuda")
    ftm.ft_linear(d, wt, x, T, y, ftm.alloc_linear_workspace(d, T), **kw)
    assert torch.all(y[T] == 7.0)      # the row behind the last is not touched
    return y[:T]


@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("T", TOKENS)
def test_linear(T, N, K):
    r = rng(T, N, K)
    wt, w = weight(r, N, K)
    for xd in (BF16, F32):
        xv, x = matrix(r, T, K, xd)
        form, q = form_of(xv)
        want, mag = q @ w.T, np.abs(q) @ np.abs(w).T
        for yd in (BF16, F32):
            y = run_linear(N, K, T, wt, x, xd, yd)
            assert_product(y, want, mag, K, yd)
            packed = run_linear(N, K, T, wt, form, ACT, yd)
            assert_product(packed, want, mag, K, yd)
            assert torch.equal(y, run_linear(N, K, T, wt, x, xd, yd))   # a fixed order of sums


@pytest.mark.parametrize("T,N,K", ((700, 1040, 1152), (260, 4096, 2176), (1000, 144, 4096), (3000, 4000, 272), (4097, 4112, 400)))
def test_linear_many_rows(T, N, K):
    """The tiled kernels, with and without a split reduction, at rows and features that end inside a tile."""
    r = rng(T, N, K)
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=1)
    form, q = form_of(xv)
    want, mag = q @ w.T, np.abs(q) @ np.abs(w).T
    for yd in (BF16, F32):
        assert_product(run_linear(N, K, T, wt, x, BF16, yd), want, mag, K, yd)
        y = torch.full((T, N), 7.0, dtype=TORCH[yd], device="cuda")
        ftm.ft_linear({"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": yd}, wt, form, T, y)   # no workspace
        assert_product(y, want, mag, K, yd)


@pytest.mark.parametrize("T,N,K", ((5, 144, 4112), (33, 144, 2064), (65, 144, 2064), (300, 144, 2064), (17, 4112, 4112),
                                   (130, 2064, 4112), (200, 2064, 8208), (777, 1040, 8208)))
def test_linear_split(T, N, K):
    """Few tiles over a long reduction: several parts, for every tile; the last block and the last tile end early."""
    r = rng(T, N, K, 13)
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=1)
    form, q = form_of(xv)
    want, mag = q @ w.T, np.abs(q) @ np.abs(w).T
    for yd in (BF16, F32):
        y = run_linear(N, K, T, wt, form, ACT, yd)
        assert_product(y, want, mag, K, yd)
        # quantised by the call: few rows take a kernel that does not split, whose sums have another order.  The
        # bound is that of any order; equal calls give equal bits.
        again = run_linear(N, K, T, wt, x, BF16, yd)
        assert_product(again, want, mag, K, yd)
        assert torch.equal(again, run_linear(N, K, T, wt, x, BF16, yd))
        assert torch.equal(y, run_linear(N, K, T, wt, form, ACT, yd))


@pytest.mark.parametrize("T,N,K", ((16, 48, 2048), (7, 272, 4592), (5, 144, 6400), (2, 1040, 16368), (1, 32, 32752), (3, 64, 10928)))
def test_linear_few_rows(T, N, K):
    """Rows that the product quantises itself: several passes over them, at the edge of what it takes and past it."""
    r = rng(T, N, K, 16)
    wt, w = weight(r, N, K)
    for xd in (BF16, F32):
        xv, x = matrix(r, T, K, xd)
        q = form_of(xv)[1]
        want, mag = q @ w.T, np.abs(q) @ np.abs(w).T
        for yd in (BF16, F32):
            y = run_linear(N, K, T, wt, x, xd, yd)
            assert_product(y, want, mag, K, yd)
            assert torch.equal(y, run_linear(N, K, T, wt, x, xd, yd))


def test_linear_long_reduction():
    """K over 512 blocks, one and many rows."""
    r = rng(5)
    N, K = 32, 65536
    wt, w = weight(r, N, K)
    for T in (1, 40):
        xv, x = matrix(r, T, K, BF16, spread=1)
        q = form_of(xv)[1]
        want, mag = q @ w.T, np.abs(q) @ np.abs(w).T
        for yd in (BF16, F32):
            assert_product(run_linear(N, K, T, wt, x, BF16, yd), want, mag, K, yd)


def test_linear_nonfinite_input_stays_in_its_row():
    r = rng(6)
    N, K, T = 64, 256, 20
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=0)
    x[3, 7], x[17, 200] = float("nan"), float("inf")
    for yd in (BF16, F32):
        for n in (4, T):
            y = run_linear(N, K, n, wt, x[:n].contiguous(), BF16, yd)
            bad = torch.isnan(y).all(dim=1).cpu()
            assert bad.tolist() == [t in (3, 17) for t in range(n)]
            assert torch.isfinite(y[~bad.cuda()]).all()


@pytest.mark.parametrize("N,K", ((16, 16), (48, 144), (128, 256), (592, 1040)))
def test_transpose(N, K):
    wt, w = weight(rng(N, K, 1), N, K)
    Np, Kp = dense.pad128(N), dense.pad128(K)
    out = {"w": torch.full((K, Np), 0xEE, dtype=torch.uint8, device="cuda"),
           "s": torch.full((Kp // 128, Np // 128), 9.0, device="cuda")}
    ftm.ft_linear_transpose(N, K, wt, out)
    got = out["w"].cpu().numpy()
    assert np.array_equal(got[:, :N], wt["w"].cpu().numpy().T[:K]) and not got[:, N:].any()
    assert torch.equal(out["s"], wt["s"].t())
    # the gradient of x over it
    T = 33
    dyv, dy = matrix(rng(N, K, 2), T, N, BF16)
    q = form_of(dyv)[1]
    for yd in (BF16, F32):
        dx = run_linear(K, N, T, out, dy, BF16, yd)
        assert_product(dx, q @ w, np.abs(q) @ np.abs(w), N, yd)


@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("T", TOKENS)
def test_weight_grad(T, N, K):
    r = rng(T, N, K, 9)
    # column forms as the quantiser leaves them (blocks run along the tokens)
    dyv, dy = matrix(r, T, N, BF16)
    xv, x = matrix(r, T, K, BF16)
    dc, xc = filled(N, T), filled(K, T)
    ftm.ft_act_quantize(dy, T, N, col=dc)
    ftm.ft_act_quantize(x, T, K, col=xc)
    a, b = form_of(dyv.T)[1], form_of(xv.T)[1]
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    for dt in (BF16, F32):
        dw = torch.full((N + 1, K), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw)
        assert torch.all(dw[N] == 3.0)
        assert_product(dw[:N], want, mag, T, dt)
    base = torch.randn(N, K, device="cuda")
    dw2 = base.clone()
    ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw2, accumulate=True)
    assert_product(dw2, want + f64(base), mag + np.abs(f64(base)), T + 1, F32)


@pytest.mark.parametrize("T,N,K", ((900, 1040, 528), (200, 4112, 4000), (5000, 272, 144)))
def test_weight_grad_of_large_weights_and_long_batches(T, N, K):
    r = rng(T, N, K, 10)
    dyv, xv = matrix(r, T, N, BF16, spread=1)[0], matrix(r, T, K, BF16, spread=1)[0]
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    for dt in (BF16, F32):
        dw = torch.full((N, K), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw)
        assert_product(dw, want, mag, T, dt)


@pytest.mark.parametrize("T,N,K", ((130, 1040, 1040), (777, 1040, 1040), (5, 2064, 2064), (300, 2064, 4112)))
def test_weight_grad_tiles(T, N, K):
    r = rng(T, N, K, 14)
    dyv, xv = matrix(r, T, N, BF16, spread=1)[0], matrix(r, T, K, BF16, spread=1)[0]
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    want, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    for dt in (BF16, F32):
        dw = torch.full((N + 1, K), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw)
        assert torch.all(dw[N] == 3.0)
        assert_product(dw[:N], want, mag, T, dt)
    ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw, accumulate=True)
    assert_product(dw[:N], 2 * want, 2 * mag, T + 1, F32)


def test_weight_grad_without_tokens():
    dw = torch.full((32, 48), 5.0, device="cuda")
    ftm.ft_linear_weight_grad(32, 48, 0, None, None, dw, accumulate=True)
    assert torch.all(dw == 5.0)
    ftm.ft_linear_weight_grad(32, 48, 0, None, None, dw)
    assert not dw.any()


# ------------------------------------------------------------------------------------- SwiGLU

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("T,I", ((1, 128), (5, 256), (127, 128), (128, 384), (130, 256), (300, 128)))
def test_swiglu(T, I, dtype):
    r = rng(T, I, 3)
    gv, gu = matrix(r, T, 2 * I, dtype, spread=1)
    h, saved, again = filled(T, I), filled(T, 2 * I), filled(T, I)
    ftm.ft_swiglu_quantize(gu, T, I, h, saved)
    assert_exact_form(saved, gv)
    assert_near_form(h, dense.swiglu(gv))
    ftm.ft_swiglu_quantize(gu, T, I, again)
    assert torch.equal(h.codes, again.codes) and torch.equal(h.scales, again.scales)

    dv, dh = matrix(r, T, I, dtype, spread=1)
    kept = form_of(gv)[1]
    d = dense.swiglu_grad(kept, dv)
    out = filled(T, 2 * I), filled(2 * I, T), filled(I, T)
    ftm.ft_swiglu_backward(saved, dh, T, I, *out)
    for c, v in zip(out, (d, d.T, dense.swiglu(kept).T)):
        assert_near_form(c, v)
    for i in range(3):
        one = [None] * 3
        one[i] = filled(out[i].rows, out[i].cols)
        ftm.ft_swiglu_backward(saved, dh, T, I, *one)
        assert torch.equal(one[i].codes, out[i].codes) and torch.equal(one[i].scales, out[i].scales)


def test_swiglu_of_far_gates():
    """Gates far below and above zero: silu vanishes or is the identity, the gradient stays finite."""
    T, I = 4, 128
    gv = np.zeros((T, 2 * I))
    gv[:, :I] = np.linspace(-3e4, 3e4, I)[None] * np.array([1, 1e-2, 1e-3, 1e30])[:, None]
    gv[:, I:] = 2.0
    gu = cuda(gv, torch.bfloat16)
    h, saved, d = filled(T, I), filled(T, 2 * I), filled(T, 2 * I)
    ftm.ft_swiglu_quantize(gu, T, I, h, saved)
    with np.errstate(over="ignore"):
        assert_near_form(h, dense.swiglu(f64(gu)))
        dh = torch.ones(T, I, dtype=torch.bfloat16, device="cuda")
        ftm.ft_swiglu_backward(saved, dh, T, I, d)
        assert_near_form(d, dense.swiglu_grad(form_of(f64(gu))[1], f64(dh)))


# ------------------------------------------------------------------------------------- router

def router_case(r, T, E, k, n_seq, padded, low=False):
    logits = r.normal(size=(T, E)) * 2
    if low:
        logits -= 120
        logits[r.random((T, E)) < 0.2] = -np.inf
        logits[::5] = -np.inf
    logits = logits.astype(np.float32)
    ids = np.argsort(-logits, axis=1, kind="stable")[:, :k].astype(np.int32)
    end = T - T // 4 if padded else T
    off = np.concatenate([[T // 8 if padded else 0], np.sort(r.integers(T // 8 if padded else 0, end + 1, n_seq - 1)), [end]]).astype(np.int32)
    mask = (r.random(T) < 0.8).astype(np.uint8) if padded else None
    return logits, ids, off, mask


def check_balance(desc, logits, ids, off, mask, pass_off=True):
    T, E = logits.shape
    out = ftm.BalanceBuffers(desc["n_seq"], E)
    for n in ("counts", "tokens"):
        getattr(out, n).fill_(77)
    for n in ("prob", "frac", "loss"):
        getattr(out, n).fill_(float("nan"))
    ws = ftm.alloc_balance_workspace(desc, T)
    ws.fill_(0xFF)
    args = dict(seq_off=cuda(off) if pass_off else None, mask=None if mask is None else cuda(mask))
    ftm.ft_balance_loss(desc, cuda(logits), cuda(ids), T, out, ws, **args)
    want = dense.balance(logits.astype(np.float64), ids, off, mask, desc["gating"], desc["coef"])
    assert np.array_equal(out.counts.cpu().numpy(), want["counts"])
    assert np.array_equal(out.tokens.cpu().numpy(), want["tokens"])
    for n in ("prob", "frac", "loss"):
        g = f64(getattr(out, n))
        assert np.all(np.abs(g - want[n]) <= 2e-5 * np.abs(want[n]) + 1e-30), n
    return out, args


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
@pytest.mark.parametrize("T,E,k,n_seq,padded", (
    (1, 1, 1, 1, False), (1, 8, 2, 1, False), (3, 5, 5, 2, False), (48, 128, 8, 1, False), (100, 60, 4, 3, True),
    (511, 256, 8, 7, True), (512, 64, 6, 1, False), (513, 64, 6, 1, False), (2000, 257, 8, 9, True),
    (3000, 1024, 64, 2, False), (700, 600, 3, 40, True), (9001, 16, 2, 300, True)))
def test_router(T, E, k, n_seq, padded, gating):
    r = rng(T, E, k, gating)
    desc = {"n_experts": E, "top_k": k, "gating": gating, "n_seq": n_seq, "coef": 0.3}
    logits, ids, off, mask = router_case(r, T, E, k, n_seq, padded)
    out, args = check_balance(desc, logits, ids, off, mask)
    sel = np.take_along_axis(logits.astype(np.float64), ids, 1)
    v = np.exp(sel - sel.max(1, keepdims=True)) if gating == oracle.GATE_SOFTMAX else dense.sigmoid(sel)
    gates = (v / v.sum(1, keepdims=True)).astype(np.float32)
    dw, dl = r.normal(size=(T, k)).astype(np.float32), r.normal(size=n_seq).astype(np.float32)
    frac = f64(out.frac)
    for use_loss, use_gates in ((True, True), (True, False), (False, True)):
        d = torch.full((T, E), 13.0, device="cuda")
        ftm.ft_router_backward(desc, cuda(logits), cuda(ids) if use_gates else None, T, out if use_loss else None,
                               cuda(dl) if use_loss else None, d, topk_w=cuda(gates) if use_gates else None,
                               d_topk_w=cuda(dw) if use_gates else None, **args)
        want, mag = dense.router_grad(logits.astype(np.float64), ids, gates.astype(np.float64), dw.astype(np.float64) if use_gates else None,
                                      off, mask, gating, frac, dl.astype(np.float64) if use_loss else None)
        got = f64(d)
        outside = np.isnan(want)
        assert np.all(got[outside] == 13.0)
        assert np.all(np.abs(got - want)[~outside] <= 2e-5 * mag[~outside] + 1e-30)


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
def test_router_far_and_infinite_logits(gating):
    """Logits whose sigmoids vanish in float32, experts at -inf, tokens with nothing but -inf."""
    r = rng(11, gating)
    for T in (37, 600):
        desc = {"n_experts": 40, "top_k": 3, "gating": gating, "n_seq": 2, "coef": 1.0}
        logits, ids, off, mask = router_case(r, T, 40, 3, 2, False, low=True)
        out, args = check_balance(desc, logits, ids, off, mask)
        d = torch.empty(T, 40, device="cuda")
        dl = np.array([1.0, -2.0], np.float32)
        ftm.ft_router_backward(desc, cuda(logits), None, T, out, cuda(dl), d, **args)
        want, mag = dense.router_grad(logits.astype(np.float64), ids, None, None, off, mask, gating, f64(out.frac), dl.astype(np.float64))
        assert np.all(np.abs(f64(d) - want) <= 2e-5 * mag + 1e-30)


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
def test_router_padding_that_is_not_finite(gating):
    """Masked tokens whose logits are NaN or infinite change nothing, and their rows of the gradient are zeros
    where the gates' gradients are."""
    r = rng(15, gating)
    for T, E in ((40, 48), (700, 200)):
        desc = {"n_experts": E, "top_k": 3, "gating": gating, "n_seq": 2, "coef": 1.0}
        logits, ids, off, _ = router_case(r, T, E, 3, 2, False)
        mask = (r.random(T) < 0.7).astype(np.uint8)
        mask[:2] = 1, 0
        bad = logits.copy()
        bad[mask == 0] = r.choice(np.float32([np.nan, np.inf, -np.inf, 3e38]), size=(int((mask == 0).sum()), E))
        gates = r.random((T, 3)).astype(np.float32)
        dw = (r.normal(size=(T, 3)) * mask[:, None]).astype(np.float32)
        grads = []
        for l in (logits, bad):
            out, args = check_balance(desc, logits, ids, off, mask)
            again = ftm.BalanceBuffers(2, E)
            ftm.ft_balance_loss(desc, cuda(l), cuda(ids), T, again, ftm.alloc_balance_workspace(desc, T), **args)
            for n in ("counts", "tokens", "prob", "frac", "loss"):
                assert torch.equal(getattr(out, n), getattr(again, n))
            d = torch.empty(T, E, device="cuda")
            ftm.ft_router_backward(desc, cuda(l), cuda(ids), T, out, torch.ones(2, device="cuda"), d, topk_w=cuda(gates),
                                   d_topk_w=cuda(dw), **args)
            grads.append(d)
        assert torch.equal(*grads) and not grads[0][torch.from_numpy(mask == 0).cuda()].any()


def test_balance_edges():
    """No tokens, empty sequences, a mask that leaves a sequence nothing, ids outside the experts, and
    one sequence without offsets."""
    r = rng(12)
    desc = {"n_experts": 8, "top_k": 2, "gating": 0, "n_seq": 4, "coef": 1.0}
    for T in (40, 640):
        logits, ids, _, _ = router_case(r, T, 8, 2, 1, False)
        ids[::3, 0], ids[1::3, 1] = -1, 8
        mask = np.ones(T, np.uint8)
        mask[10:20] = 0
        out, args = check_balance(desc, logits, ids, np.array([0, 10, 20, 20, T], np.int32), mask)
        d = torch.full((T, 8), 2.0, device="cuda")
        dl = torch.ones(4, device="cuda")
        ftm.ft_router_backward(desc, cuda(logits), None, T, out, dl, d, **args)
        assert not d[10:20].any() and torch.isfinite(d).all()
        check_balance(dict(desc, n_seq=1), logits, ids, np.array([0, T]), None, pass_off=False)
    zero, _ = check_balance(dict(desc, n_seq=1), np.zeros((0, 8), np.float32), np.zeros((0, 2), np.int32), np.array([0, 0]), None, pass_off=False)
    assert not zero.counts.any()


# ------------------------------------------------------------------------- together, and in use

def expert_step(x, dy, W13, W13t, W2, W2t, T, H, I, B):
    """Forward and backward pass of a dense SwiGLU layer as a training loop runs it."""
    lin = lambda o, i, xd=ACT, yd=BF16: {"out_features": o, "in_features": i, "x_dtype": xd, "y_dtype": yd}
    ftm.ft_act_quantize(x, T, H, B["x"], B["x_col"])
    ftm.ft_linear(lin(2 * I, H), W13, B["x"], T, B["gu"])
    ftm.ft_swiglu_quantize(B["gu"], T, I, B["h"], B["saved"])
    ftm.ft_linear(lin(H, I, yd=F32), W2, B["h"], T, B["y"])
    ftm.ft_act_quantize(dy, T, H, B["dy"], B["dy_col"])
    ftm.ft_linear(lin(I, H), W2t, B["dy"], T, B["dh"])
    ftm.ft_swiglu_backward(B["saved"], B["dh"], T, I, B["dgu"], B["dgu_col"], B["h_col"])
    ftm.ft_linear(lin(H, 2 * I), W13t, B["dgu"], T, B["dx"])
    ftm.ft_linear_weight_grad(H, I, T, B["dy_col"], B["h_col"], B["dw2"])
    ftm.ft_linear_weight_grad(2 * I, H, T, B["dgu_col"], B["x_col"], B["dw13"])
    return {n: B[n] for n in ("y", "dx", "dw2", "dw13")}


def expert_buffers(T, H, I):
    A, e = ftm.ActCodes, lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt, device="cuda")
    return {"x": A(T, H), "x_col": A(H, T), "gu": e(T, 2 * I), "h": A(T, I), "saved": A(T, 2 * I),
            "y": e(T, H, dt=torch.float32), "dy": A(T, H), "dy_col": A(H, T), "dh": e(T, I), "dgu": A(T, 2 * I),
            "dgu_col": A(2 * I, T), "h_col": A(I, T), "dx": e(T, H), "dw2": e(H, I, dt=torch.float32),
            "dw13": e(2 * I, H, dt=torch.float32)}


def expert_weights(r, H, I):
    def one(N, K):
        v = r.normal(size=(N, K)) / np.sqrt(K)
        s = np.abs(v.reshape(N // 128, 128, K // 128, 128)).max(axis=(1, 3)) / 448
        s = s.astype(np.float32)
        w = dense.nearest_code(np.clip(v / np.repeat(np.repeat(s, 128, 0), 128, 1), -448, 448))
        wt = {"w": torch.empty(K, N, dtype=torch.uint8, device="cuda"), "s": torch.empty(K // 128, N // 128, device="cuda")}
        fwd = {"w": cuda(w), "s": cuda(s)}
        ftm.ft_linear_transpose(N, K, fwd, wt)
        return fwd, wt, dense.weight_values(w, s)
    return one(2 * I, H), one(H, I)


def normwise(got, want):
    return np.linalg.norm(f64(got) - want) / np.linalg.norm(want)


def test_expert_step_against_64_bits():
    """The operators together: a dense SwiGLU layer's step.  Against the same layer in 64 bits with no
    8-bit activations at all, every quantisation (2^-4 at most, about 2^-5.5 on average over a step) enters
    the results once per operand: two or three of them give some 5 percent normwise, 10 are allowed."""
    T, H, I = 200, 256, 128
    r = rng(21)
    (W13, W13t, w13), (W2, W2t, w2) = expert_weights(r, H, I)
    x, dy = cuda(r.normal(size=(T, H)), torch.bfloat16), cuda(r.normal(size=(T, H)) * 1e-4, torch.bfloat16)
    out = expert_step(x, dy, W13, W13t, W2, W2t, T, H, I, expert_buffers(T, H, I))
    X, D = f64(x), f64(dy)
    gu = X @ w13.T
    h = dense.swiglu(gu)
    dgu = dense.swiglu_grad(gu, D @ w2)
    want = {"y": h @ w2.T, "dx": dgu @ w13, "dw2": D.T @ h, "dw13": dgu.T @ X}
    for n, v in want.items():
        assert normwise(out[n], v) < 0.1, n


def test_expert_step_replayed_and_on_a_side_stream():
    """Captured once on a side stream and replayed with new inputs, eager work between the replays; every
    replay equals the eager step."""
    T, H, I = 130, 256, 128
    r = rng(22)
    (W13, W13t, _), (W2, W2t, _) = expert_weights(r, H, I)
    x, dy = torch.empty(T, H, dtype=torch.bfloat16, device="cuda"), torch.empty(T, H, dtype=torch.bfloat16, device="cuda")
    B, B2 = expert_buffers(T, H, I), expert_buffers(T, H, I)
    args = (x, dy, W13, W13t, W2, W2t, T, H, I)
    side = torch.cuda.Stream()
    x.normal_()
    dy.normal_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        expert_step(*args, B)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        out = expert_step(*args, B)
    for i in range(4):
        x.normal_()
        dy.normal_()
        for v in out.values():
            v.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = {n: v.clone() for n, v in out.items()}
        want = expert_step(*args, B2)
        for n in want:
            assert torch.equal(got[n], want[n]), (i, n)


def test_router_step_after_the_layer_call():
    """Routing by ft_route_only, its balance loss, and the gradient back to the logits, captured and
    replayed."""
    T, E, k, H = 700, 64, 6, 256
    desc = dict(hidden=H, inter=128, n_experts=E, top_k=k, gating=1, w_dtype=BF16, x_dtype=BF16, n_slots=0, shared_slot=-1)
    bd = {"n_experts": E, "top_k": k, "gating": 1, "n_seq": 2, "coef": 0.01}
    logits = torch.empty(T, E, device="cuda")
    table = torch.full((E,), -1, dtype=torch.int32, device="cuda")
    route, ws = ftm.RouteBuffers(T, k, E), ftm.alloc_workspace(desc, T)
    out, bws = ftm.BalanceBuffers(2, E), ftm.alloc_balance_workspace(bd, T)
    off = torch.tensor([0, 300, 650], dtype=torch.int32, device="cuda")
    dl, dw, d = torch.ones(2, device="cuda"), torch.randn(T, k, device="cuda"), torch.zeros(T, E, device="cuda")

    def step():
        ftm.ft_route_only(desc, logits, table, T, route, ws)
        ftm.ft_balance_loss(bd, logits, route.topk_ids, T, out, bws, seq_off=off)
        ftm.ft_router_backward(bd, logits, route.topk_ids, T, out, dl, d, topk_w=route.topk_w, d_topk_w=dw, seq_off=off)

    logits.normal_()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(3):
        logits.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = d.clone(), out.loss.clone(), out.counts.clone()
        l, ids = f64(logits), route.topk_ids.view(T, k).cpu().numpy()
        want = dense.balance(l, ids, [0, 300, 650], None, 1, 0.01)
        assert np.array_equal(got[2].cpu().numpy(), want["counts"])
        assert np.allclose(f64(got[1]), want["loss"], rtol=2e-5, atol=0)
        g, mag = dense.router_grad(l, ids, f64(route.topk_w).reshape(T, k), f64(dw), [0, 300, 650], None, 1, f64(out.frac), f64(dl))
        assert np.all(np.abs(f64(got[0]) - g)[:650] <= 2e-5 * mag[:650] + 1e-30) and not got[0][650:].any()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], d) and torch.equal(got[1], out.loss)


def test_calls_with_workspaces_captured_and_at_once():
    """Few rows, a split reduction, and the balance loss in parts, with their workspaces: captured and replayed with
    new inputs and eager work between the replays, and on two streams at once, every result the eager call's bits."""
    r = rng(23)
    N, K, E, k, n_seq, Tb = 528, 4112, 48, 4, 5, 2000
    wt, _ = weight(r, N, K)
    desc = lambda xd: {"out_features": N, "in_features": K, "x_dtype": xd, "y_dtype": BF16}
    bal = {"n_experts": E, "top_k": k, "gating": 1, "n_seq": n_seq, "coef": 0.5}
    off = cuda(np.array([0, 400, 400, 900, 1700, 1900], np.int32))

    def state():
        return {"few": torch.empty(3, K, dtype=torch.bfloat16, device="cuda"), "many": torch.empty(150, K, dtype=torch.bfloat16, device="cuda"),
                "logits": torch.empty(Tb, E, device="cuda"), "ids": torch.empty(Tb, k, dtype=torch.int32, device="cuda"),
                "y3": torch.zeros(3, N, dtype=torch.bfloat16, device="cuda"), "y150": torch.zeros(150, N, dtype=torch.bfloat16, device="cuda"),
                "d": torch.zeros(Tb, E, device="cuda"), "out": ftm.BalanceBuffers(n_seq, E), "one": torch.ones(n_seq, device="cuda"),
                "ws": ftm.alloc_linear_workspace(desc(BF16), 150), "bws": ftm.alloc_balance_workspace(bal, Tb)}

    def fill(s, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for n in ("few", "many", "logits"):
            s[n].normal_(generator=g)
        s["ids"].copy_(s["logits"].topk(k, dim=1).indices)

    def run(s):
        ftm.ft_linear(desc(BF16), wt, s["few"], 3, s["y3"], s["ws"])
        ftm.ft_linear(desc(BF16), wt, s["many"], 150, s["y150"], s["ws"])
        ftm.ft_balance_loss(bal, s["logits"], s["ids"], Tb, s["out"], s["bws"], seq_off=off)
        ftm.ft_router_backward(bal, s["logits"], None, Tb, s["out"], s["one"], s["d"], seq_off=off)

    results = lambda s: [s["y3"], s["y150"], s["d"], s["out"].loss, s["out"].counts, s["out"].frac]
    a, b = state(), state()
    fill(a, 0)
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run(a)
    for seed in (1, 2, 3):
        fill(a, seed)
        graph.replay()
        fill(b, seed)
        run(b)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(results(a), results(b)))
    want = [[t.clone() for t in results(b)]]
    fill(a, 4)
    run(a)
    want.append([t.clone() for t in results(a)])
    for s in (a, b):
        for t in results(s):
            t.zero_()
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(side):
            run(b)
        with torch.cuda.stream(other):
            run(a)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(results(b), want[0]))
    assert all(torch.equal(x, y) for x, y in zip(results(a), want[1]))


def test_offsets_past_32_bits():
    """1048576 tokens, all zeros but the last 384: codes, results and inputs past 4 GiB, in every form and product.
    Rows of zeros add exact zeros to a sum, so the bounds are those of 384 terms."""
    T, L, N, K = 1048576, 384, 2064, 4112
    r = rng(24)
    wt, w = weight(r, N, K)
    xv, xl = matrix(r, L, K, BF16, spread=1)
    dv, dl = matrix(r, L, N, BF16, spread=1)
    x, dy = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, N, dtype=torch.bfloat16, device="cuda")
    x[-L:], dy[-L:] = xl, dl
    row, xc, dc = ftm.ActCodes(T, K), ftm.ActCodes(K, T), ftm.ActCodes(N, T)
    ftm.ft_act_quantize(x, T, K, row, xc)
    ftm.ft_act_quantize(dy, T, N, col=dc)
    del x, dy
    codes, scales = dense.quantize(xv)
    assert np.array_equal(row.codes[-L:].cpu().numpy(), codes) and np.array_equal(row.scales[:, -L:].cpu().numpy(), scales[:, :L])
    assert not row.codes[:-L].any()
    for c, v in ((xc, xv), (dc, dv)):
        codes, scales = dense.quantize(v.T)
        assert np.array_equal(c.codes[:, -L:].cpu().numpy(), codes)
        assert np.array_equal(c.scales[-L // 128:, :v.shape[1]].cpu().numpy(), scales[:, :v.shape[1]])
    q, a, b = form_of(xv)[1], form_of(dv.T)[1], form_of(xv.T)[1]
    y = torch.full((T, N), 7.0, dtype=torch.bfloat16, device="cuda")
    ftm.ft_linear({"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": BF16}, wt, row, T, y)
    assert_product(y[-L:], q @ w.T, np.abs(q) @ np.abs(w).T, K, BF16)
    assert not y[:-L].any()
    for dt in (BF16, F32):
        dw = torch.empty(N, K, dtype=TORCH[dt], device="cuda")
        ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw)
        assert_product(dw, a @ b.T, np.abs(a) @ np.abs(b).T, L, dt)
