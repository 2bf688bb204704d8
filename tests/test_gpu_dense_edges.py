"""Edges of the dense 8-bit operators and of the router's gradient: what is not finite, factors that overflow, long sums,
and the branches that only large or odd calls take."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_16157_amd as ftm
from oracle import dense
from tests.test_gpu_dense import (ACT, BF16, F32, TORCH, assert_exact_form, assert_near_form, assert_product, cuda, f64,
                                  filled, form_of, matrix, rng, run_linear, weight)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------- weight blocks of scale 0

def zero_blocks(r, wt):
    """A third of the weight's blocks, the first and the last of a row of blocks among them, with scale 0: the weight
    with codes 0 there, and with NaN codes."""
    zero = r.random(tuple(wt["s"].shape)) < 1 / 3
    zero[0, 0] = zero[-1, -1] = True
    codes = np.repeat(np.repeat(zero, 128, 0), 128, 1)[:wt["w"].shape[0]]
    w, s = wt["w"].cpu().numpy(), wt["s"].cpu().numpy()
    s[zero] = 0
    out = []
    for code in (0, r.choice(np.uint8([0x7F, 0xFF]), size=w.shape)):
        out.append({"w": cuda(np.where(codes, code, w).astype(np.uint8)), "s": cuda(s)})
    return out


@pytest.mark.parametrize("T,N,K", ((1, 272, 1040), (3, 4432, 1168), (16, 272, 1040), (33, 272, 1040), (40, 144, 2064),
                                   (130, 528, 2064), (300, 272, 1040), (777, 1552, 2064), (197, 4192, 4384),
                                   (1922, 4256, 800)))
def test_linear_blocks_of_scale_0(T, N, K):
    """They add nothing, whatever their codes hold: the same bits as with codes 0, in every kernel, with and without
    a split reduction, and in the gradient of x over the transposed weight."""
    r = rng(T, N, K, 30)
    clean, nan = zero_blocks(r, weight(r, N, K)[0])
    xv, x = matrix(r, T, K, BF16, spread=1)
    form = form_of(xv)[0]
    for yd in (BF16, F32):
        want = run_linear(N, K, T, clean, x, BF16, yd)
        assert torch.isfinite(want).all()
        assert torch.equal(run_linear(N, K, T, nan, x, BF16, yd), want)
        assert torch.equal(run_linear(N, K, T, nan, form, ACT, yd), run_linear(N, K, T, clean, form, ACT, yd))
        d = {"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": yd}
        whole = [torch.empty(T, N, dtype=TORCH[yd], device="cuda") for _ in range(2)]
        for wt, y in zip((clean, nan), whole):
            ftm.ft_linear(d, wt, form, T, y)   # no workspace: not split
        assert torch.equal(*whole)
    back = []
    for wt in (clean, nan):
        t = {"w": torch.empty(K, dense.pad128(N), dtype=torch.uint8, device="cuda"),
             "s": torch.empty(dense.pad128(K) // 128, dense.pad128(N) // 128, device="cuda")}
        ftm.ft_linear_transpose(N, K, wt, t)
        back.append(run_linear(K, N, T, t, want, F32, BF16))
    assert torch.equal(*back) and torch.isfinite(back[0]).all()


@pytest.mark.parametrize("T,N,K", ((4, 144, 1040), (20, 144, 1040), (300, 272, 1040), (1922, 4256, 800)))
def test_linear_blocks_of_scale_0_meet_what_is_not_finite(T, N, K):
    """Nor does it matter what x holds there: an infinity or NaN in channels all of whose weight blocks have scale 0
    changes nothing."""
    r = rng(T, N, K, 31)
    wt = weight(r, N, K)[0]
    wt["s"][:, 2] = 0
    x = torch.randn(T, K, generator=torch.Generator().manual_seed(T)).to("cuda", torch.bfloat16)
    bad = x.clone()
    x[::3, 300] = 0.0
    bad[::3, 300] = float("nan")
    bad[::6, 300] = float("inf")
    for yd in (BF16, F32):
        want = run_linear(N, K, T, wt, x, BF16, yd)
        assert torch.isfinite(want).all() and torch.equal(run_linear(N, K, T, wt, bad, BF16, yd), want)


# ----------------------------------------------------------------------------- signalling NaNs

@pytest.mark.parametrize("dtype", (BF16, F32))
@pytest.mark.parametrize("T,C", ((40, 256), (130, 400), (257, 128)))
def test_signalling_nans_leave_their_block_its_scale(T, C, dtype):
    """Signalling NaNs anywhere in a block, in front of, behind and between values of many magnitudes: NaN codes, and
    the scale and the other codes those of the block without them."""
    r = rng(T, C, dtype, 32)
    x = (r.normal(size=(T, C)) * 10.0 ** r.uniform(-3, 3, (T, C))).astype(np.float32)
    if dtype == BF16:
        bits = (x.view(np.uint32) >> 16).astype(np.uint16)
        snan, quiet = np.uint16([0x7F81, 0xFFBF]), np.uint16([0x7FC0, 0xFFC1])
    else:
        bits = x.view(np.uint32).copy()
        snan, quiet = np.uint32([0x7F800001, 0xFFBFFFFF]), np.uint32([0x7FC00000, 0xFFC00001])
    at = r.random((T, C)) < 0.1
    bits[at] = r.choice(snan, size=int(at.sum()))
    bits[0, :128] = snan[0]
    bits[1, :127] = snan[1]   # one value of its block left
    some = r.random((T, C)) < 0.02
    bits[some] = r.choice(quiet, size=int(some.sum()))
    x = (bits.astype(np.uint32) << 16 if dtype == BF16 else bits).view(np.float32)
    t = torch.from_numpy(bits.view(np.int16 if dtype == BF16 else np.int32)).cuda().view(TORCH[dtype])

    def check(c, v):
        with np.errstate(invalid="ignore"):
            codes, s = dense.quantize(v.astype(np.float64))
        got = c.codes.cpu().numpy()
        nan = (codes & 0x7F) == 0x7F
        assert np.array_equal(c.scales.cpu().numpy()[:, :v.shape[0]], s)
        assert np.array_equal((got & 0x7F) == 0x7F, nan) and np.array_equal(got[~nan], codes[~nan])

    row, col, alone = filled(T, C), filled(C, T), filled(T, C)
    ftm.ft_act_quantize(t, T, C, row, col)
    ftm.ft_act_quantize(t, T, C, alone)
    check(alone, x)
    check(row, x)
    check(col, x.T)
    if C % 256 == 0:   # kept by SwiGLU
        h, saved = filled(T, C // 2), filled(T, C)
        ftm.ft_swiglu_quantize(t, T, C // 2, h, saved)
        check(saved, x)


def test_signalling_nans_inside_the_product():
    """Rows that the product quantises itself: the other rows are not touched, and a row's NaNs that meet only weight
    blocks of scale 0 leave the row's other blocks as they are."""
    T, N, K = 4, 64, 512
    r = rng(33)
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=1)
    x.view(torch.int16)[1, 200] = 0x7F81
    x.view(torch.int16)[1, 130] = -1          # a quiet one
    y = run_linear(N, K, T, wt, x, BF16, F32)
    q = form_of(np.where(np.isfinite(f64(x)), f64(x), 0.0))[1]
    keep = [0, 2, 3]
    assert_product(y[keep], q[keep] @ w.T, np.abs(q[keep]) @ np.abs(w).T, K, F32)
    wt["s"][:, 1], w[:, 128:256] = 0, 0
    assert_product(run_linear(N, K, T, wt, x, BF16, F32), q @ w.T, np.abs(q) @ np.abs(w).T, K, F32)


# ------------------------------------------------------------------------------ SwiGLU backward

@pytest.mark.parametrize("gate", (-60.0, -144.0))
def test_swiglu_gradient_whose_factors_overflow(gate):
    """dh up past float32's largest value where the sigmoid brings the gradient back: d_gate is finite, and no NaN code
    is left.  At gate -60 every element of a block is such a product; at -144, where the sigmoid is 0 in float32, one in
    a block of ordinary ones."""
    T, I = 3, 128
    gv, dv = np.ones((T, 2 * I)), np.full((T, I), 2.0 ** -100)
    gv[:, I:] = 2.0 ** 100
    cols = slice(0, I) if gate == -60.0 else slice(5, 6)
    gv[:, cols], dv[:, cols] = gate, 2.0 ** 40
    saved, kept = form_of(gv)
    assert np.array_equal(kept, gv)
    want = dense.swiglu_grad(gv, dv)
    assert np.isfinite(want).all() and np.abs(want).max() < 1e37
    for dtype in (BF16, F32):
        row, col = filled(T, 2 * I), filled(2 * I, T)
        ftm.ft_swiglu_backward(saved, cuda(dv).to(TORCH[dtype]), T, I, row, col)
        assert_near_form(row, want)
        codes = col.codes.cpu().numpy()
        assert not ((codes & 0x7F) == 0x7F).any()
        if gate == -60.0:
            assert_near_form(col, want.T)


# ---------------------------------------------------------------------------------- long sums

@pytest.mark.parametrize("T,E", ((511, 7), (8191, 300), (20011, 300), (100003, 131), (100003, 1000), (1000003, 11)))
def test_balance_sums_do_not_drift(T, E):
    """Equal logits: every probability is the same float32, the rounded 1 / E, and its sum over the tokens must stay
    exact but for roundings that do not grow with the tokens: one of each wave's sum, one of each part's and one of
    the result, 2^-24 of it each as all terms are positive.  (A float32 running sum of equal terms is off by tens of
    such steps.)  frac is exact to its rounding, and the loss has one more rounding."""
    desc = {"n_experts": E, "top_k": 1, "gating": 0, "n_seq": 1, "coef": 1.0}
    ids = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    out = ftm.BalanceBuffers(1, E)
    ftm.ft_balance_loss(desc, torch.zeros(T, E, device="cuda"), ids, T, out, ftm.alloc_balance_workspace(desc, T))
    p = float(np.float32(1) / np.float32(E))
    assert np.all(np.abs(f64(out.prob) - p) <= 3 * 2.0 ** -24 * p)
    assert np.array_equal(f64(out.frac)[0], [E] + [0] * (E - 1))
    assert abs(f64(out.loss)[0] - p * E) <= 4 * 2.0 ** -24 * p * E
    assert out.tokens.item() == T and out.counts[0, 0].item() == T


# ------------------------------------------------------------------------- branches of the router

def router_both_ways(desc, logits, ids, off, mask, r):
    """Forward and backward against the oracle, with the bounds of the module these helpers come from."""
    T, E, k, n_seq, gating = *logits.shape, desc["top_k"], desc["n_seq"], desc["gating"]
    out = ftm.BalanceBuffers(n_seq, E)
    args = dict(seq_off=cuda(off), mask=None if mask is None else cuda(mask))
    ftm.ft_balance_loss(desc, cuda(logits), cuda(ids), T, out, ftm.alloc_balance_workspace(desc, T), **args)
    l64 = logits.astype(np.float64)
    want = dense.balance(l64, ids, off, mask, gating, desc["coef"])
    assert np.array_equal(out.counts.cpu().numpy(), want["counts"])
    assert np.array_equal(out.tokens.cpu().numpy(), want["tokens"])
    for n in ("prob", "frac", "loss"):
        assert np.all(np.abs(f64(getattr(out, n)) - want[n]) <= 2e-5 * np.abs(want[n]) + 1e-30), n
    sel = np.take_along_axis(l64, np.clip(ids, 0, E - 1), 1)
    v = np.exp(sel - sel.max(1, keepdims=True)) if gating == oracle.GATE_SOFTMAX else dense.sigmoid(sel)
    gates = (v / v.sum(1, keepdims=True)).astype(np.float32)
    dw, dl = r.normal(size=(T, k)).astype(np.float32), r.normal(size=n_seq).astype(np.float32)
    d = torch.full((T, E), 13.0, device="cuda")
    ftm.ft_router_backward(desc, cuda(logits), cuda(ids), T, out, cuda(dl), d, topk_w=cuda(gates), d_topk_w=cuda(dw), **args)
    g, mag = dense.router_grad(l64, ids, gates.astype(np.float64), dw.astype(np.float64), off, mask, gating, f64(out.frac),
                               dl.astype(np.float64))
    got, outside = f64(d), np.isnan(g)
    assert outside.any() == (off[0] > 0 or off[-1] < T) and np.all(got[outside] == 13.0)
    assert np.all(np.abs(got - g)[~outside] <= 2e-5 * mag[~outside] + 1e-30)


def router_inputs(r, T, E, k):
    logits = (r.normal(size=(T, E)) * 2).astype(np.float32)
    return logits, np.argsort(-logits, axis=1, kind="stable")[:, :k].astype(np.int32)


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
@pytest.mark.parametrize("T,E,k,n_seq", ((16385, 48, 5, 300), (20003, 128, 17, 40), (16387, 256, 8, 300), (17001, 320, 33, 64),
                                         (16384, 64, 2, 1)))
def test_router_of_many_tokens_and_short_sequences(T, E, k, n_seq, gating):
    """Runs of four tokens a lane row: sequences of none to three tokens, so that several end inside a run, long ones
    around them, tokens of none at both ends, a last run that is not whole."""
    r = rng(T, E, gating, 34)
    if n_seq > 1:
        short = r.integers(0, 4, n_seq - 3)
        first, middle = 1021, T // 2 + 1     # no multiples of a run
        off = np.concatenate([[first, middle], middle + np.cumsum(short), [T - 1500, T - 7]]).astype(np.int32)
    else:
        off = np.array([0, T], np.int32)
    assert len(off) == n_seq + 1 and np.all(np.diff(off) >= 0)
    mask = (r.random(T) < 0.8).astype(np.uint8)
    logits, ids = router_inputs(r, T, E, k)
    router_both_ways({"n_experts": E, "top_k": k, "gating": gating, "n_seq": n_seq, "coef": 0.3}, logits, ids, off, mask, r)


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
@pytest.mark.parametrize("E,k", ((64, 17), (64, 33), (64, 64), (128, 17), (128, 48), (100, 64)))
@pytest.mark.parametrize("T", (1, 130, 700))
def test_router_of_more_experts_a_token_than_lanes(T, E, k, gating):
    """Up to 128 experts a token has 16 lanes: with more selected ones each lane holds several."""
    r = rng(T, E, k, gating, 35)
    off = np.array([0, T // 3, T], np.int32)
    logits, ids = router_inputs(r, T, E, k)
    if T > 1:
        ids[::7, k - 1], ids[1::7, 16] = -1, E     # not counted
    router_both_ways({"n_experts": E, "top_k": k, "gating": gating, "n_seq": 2, "coef": 0.3}, logits, np.ascontiguousarray(ids),
                     off, None, r)


# ------------------------------------------------------------------ the 256 x 256 tile, dense data

@pytest.mark.parametrize("T,N,K", ((1922, 4256, 800), (2500, 4112, 1808)))
def test_linear_of_the_largest_tile(T, N, K):
    """7 and 15 blocks of reduction, so that every place of the tile's rings is filled more than once; rows, features
    and the last block end inside a tile."""
    r = rng(T, N, K, 36)
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=1)
    form, q = form_of(xv)
    y = run_linear(N, K, T, wt, x, BF16, BF16)
    assert_product(y, q @ w.T, np.abs(q) @ np.abs(w).T, K, BF16)
    assert torch.equal(y, run_linear(N, K, T, wt, form, ACT, BF16))


@pytest.mark.parametrize("T,N,K", ((803, 6800, 1168), (1000, 4096, 4096), (2004, 4752, 1936)))
def test_weight_grad_of_the_largest_tile(T, N, K):
    r = rng(T, N, K, 37)
    dyv, xv = matrix(r, T, N, BF16, spread=1)[0], matrix(r, T, K, BF16, spread=1)[0]
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    dw = torch.full((N + 1, K), 3.0, dtype=torch.bfloat16, device="cuda")
    ftm.ft_linear_weight_grad(N, K, T, dc, xc, dw)
    assert torch.all(dw[N] == 3.0)
    assert_product(dw[:N], a @ b.T, np.abs(a) @ np.abs(b).T, T, BF16)


def test_linear_of_the_largest_tile_split():
    """A reduction long enough that even this tile's is split: 129 blocks in 7 parts."""
    T, N, K = 132, 8272, 16496
    r = rng(38)
    wt, w = weight(r, N, K)
    xv, x = matrix(r, T, K, BF16, spread=1)
    form, q = form_of(xv)
    y = run_linear(N, K, T, wt, form, ACT, BF16)
    assert_product(y, q @ w.T, np.abs(q) @ np.abs(w).T, K, BF16)
    assert torch.equal(y, run_linear(N, K, T, wt, form, ACT, BF16))


# --------------------------------------------------------------- sums of the fp8 matrix instructions

def fp8_sum_bound(a, b, scale):
    """How far the fp8 instructions' sums of a [T][K] times b [N][K] may be off (values of codes, one scale for all):
    within each group of 8 channels the products lose what lies below 2^-13 of the largest one's power of two, where a
    code below 2^-6 (subnormal, or 0) counts as 2^-6; the groups' sums then add up in float32 (16 a block, and one
    a block)."""
    ex = lambda v: np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -20))), -6)
    pad = lambda v: np.pad(v, ((0, 0), (0, -v.shape[1] % 8)))
    ea, eb = ex(pad(a)).reshape(len(a), 1, -1, 8), ex(pad(b)).reshape(1, len(b), -1, 8)
    lost = np.concatenate([(8 * 2.0 ** ((ea[t:t + 4] + eb).max(axis=3) - 13)).sum(axis=2) for t in range(0, len(a), 4)])
    return scale * (lost + 2.0 ** -24 * (16 + a.shape[1] / 128 + 2) * (np.abs(a) @ np.abs(b).T))


@pytest.mark.parametrize("T,N,K", ((5, 144, 1040), (40, 144, 2064), (300, 272, 528)))
@pytest.mark.parametrize("kind", ("spread", "cancel", "small among large", "subnormal"))
def test_products_where_the_sum_is_small_against_its_terms(T, N, K, kind):
    """bf16 results are bounded by the fp8 instructions' own rule, not by the result: magnitudes that span 2^17, terms
    that cancel in pairs, one large term and many just below what is kept, large terms that come from subnormal
    codes.  float32 results keep float32's bound."""
    r = rng(T, N, K, 39)
    sign = lambda *s: np.where(r.random(s) < 0.5, -1.0, 1.0)
    if kind == "small among large":
        x, w = np.full((T, K), 2.75), np.full((N, K), 2.75)     # 7.6 next to 256 * 256: nothing of it is kept
        x[:, ::8], w[:, ::8] = 256.0, 256.0
        w[:, ::16] *= -1
    elif kind == "subnormal":
        x, w = np.full((T, K), 0.078125), np.full((N, K), 0.0546875)
        x[:, ::8], w[:, ::8] = 2.0 ** -9, 256.0
        x[:, 5::16], w[:, 5::16] = 256.0, -(2.0 ** -9)
    else:
        x, w = sign(T, K) * 2.0 ** r.uniform(-8, 8, (T, K)), sign(N, K) * 2.0 ** r.uniform(-8, 8, (N, K))
        if kind == "cancel":
            x[:, 1::2], w[:, 1::2] = -x[:, ::2], w[:, ::2] * np.where(r.random((N, K // 2)) < 0.9, 1.0, 1.125)
    x[:, :16] = np.where(np.arange(16) == 0, 448.0, x[:, :16])      # so that every block's scale is 1
    x[:, 128::128] = 448.0
    codes = np.zeros((N, dense.pad128(K)), np.uint8)
    codes[:, :K] = dense.nearest_code(w)
    codes[:, ::128] = 0
    wt = {"w": cuda(codes), "s": torch.full((dense.pad128(N) // 128, codes.shape[1] // 128), 0.75, device="cuda")}
    wv = dense._VALUES[codes][:, :K]
    form, q = form_of(x)
    assert torch.all(form.scales[:, :T] == 127)
    want, mag = 0.75 * (q @ wv.T), 0.75 * (np.abs(q) @ np.abs(wv).T)
    y = f64(run_linear(N, K, T, wt, form, ACT, BF16))
    assert np.all(np.abs(y - want) <= 2.0 ** -8 * np.abs(want) + (1 + 2.0 ** -8) * fp8_sum_bound(q, wv, 0.75))
    assert_product(run_linear(N, K, T, wt, form, ACT, F32), want, mag, K, F32)
