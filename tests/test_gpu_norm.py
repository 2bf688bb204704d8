"""The norms before and after a block on the GPU against the 64-bit oracle.

Tolerances, from the arithmetic (u = 2^-24).  A row's sum of squares has positive terms and goes through at most 8 CH + 24
additions (CH <= 8 runs of 8 channels a thread, 6 across the lanes, 16 across the waves), so 1/rms is off by at most
50 u; a product of up to six factors adds 6 u.  So
* r: 60 u of the step's magnitude and one rounding of the sum;
* n: 120 u of pre (|x| + |step|) / rms(r), since r's error enters once itself and once, averaged, through rms(r);
* gradients: every term is such a product, and sums over a token or over T tokens of terms of either sign add at most
  (T or 90) u of the sum of magnitudes: 400 u of the magnitudes the oracle sums up for those of a token, (400 + T) u for
  those over the tokens;
then one rounding to the output's type.  For channels of up to 65536 within float32's range.
"""
import numpy as np
import pytest
import torch

import paper_2608_16157_amd as ftm
from oracle import dense, experts
from tests.test_gpu_dense import BF16, F32, TORCH, assert_near_form, cuda, f64, filled, rng

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NAMES = ("pre", "post", "gate", "token_gate")


def half(kind):
    return 2.0 ** -8 if kind == BF16 else U


def tensor(r, shape, kind, size=1.0):
    t = cuda(r.normal(size=shape) * size).to(TORCH[kind])
    return f64(t), t


def inputs(r, T, C, xt, yt, wt, post, left_out=()):
    d = {"channels": C, "x_dtype": xt, "y_dtype": yt, "w_dtype": wt, "post_norm": post, "eps": 1e-5, "scale": -0.75}
    val, dev = {}, {}
    for n in NAMES:
        shape, kind = (T, F32) if n == "token_gate" else (C, wt)
        val[n], dev[n] = (np.ones(shape), None) if n in left_out else tensor(r, shape, kind)
    return d, val, dev


def rows(r, T, C, kind):
    """Rows of different sizes."""
    t = cuda(r.normal(size=(T, C)) * 10.0 ** r.uniform(-2, 2, (T, 1))).to(TORCH[kind])
    return f64(t), t


def forward_tolerance(d, val, x, b):
    step = np.zeros_like(x)
    if b is not None:
        u = val["post"] * b / experts._rms(b, d["eps"]) if d["post_norm"] else b
        step = np.abs(d["scale"] * val["gate"] * val["token_gate"][:, None] * u)
    return step


def check_forward(d, val, dev, x, b, T, out):
    """x, b: (values, tensor) or b None; out: the types asked for."""
    C, xt, yt = d["channels"], d["x_dtype"], d["y_dtype"]
    r_t = torch.full((T + 1, C), 7.0, dtype=TORCH[xt], device="cuda") if "r" in out else None
    n_t = torch.full((T + 1, C), 7.0, dtype=TORCH[yt], device="cuda") if "n" in out else None
    form = filled(T, C) if "row" in out else None
    ftm.ft_block_norm(d, dev, x[1], None if b is None else b[1], T, r_t, n_t, form)
    bv = None if b is None else b[0]
    rv, nv = experts.norm(x[0], bv, post_norm=d["post_norm"], eps=d["eps"], scale=d["scale"], **val)
    step = forward_tolerance(d, val, x[0], bv)
    mag = np.abs(val["pre"]) * (np.abs(x[0]) + step) / experts._rms(rv, d["eps"])
    # what of r's own error comes back through rms(r), relative to r
    back = 1 + np.sqrt(((np.abs(x[0]) + step) ** 2).mean(axis=1, keepdims=True)) / experts._rms(rv, d["eps"])
    if r_t is not None and b is not None:
        assert np.all(np.abs(f64(r_t[:T]) - rv) <= half(xt) * np.abs(rv) + 61 * U * (step + np.abs(rv)))
        assert torch.all(r_t[T] == 7.0)
    if n_t is not None:
        assert np.all(np.abs(f64(n_t[:T]) - nv) <= half(yt) * np.abs(nv) + 121 * U * mag * back)
        assert torch.all(n_t[T] == 7.0)
    if form is not None:
        assert_near_form(form, nv)
    return r_t, n_t, form


# one class of sizes after the other, ends inside a class, one lane row, partial blocks of 128
SIZES = ((1, 16), (3, 48), (2, 128), (130, 144), (33, 512), (9, 528), (5, 1024), (7, 1040), (17, 2048), (3, 2064), (2, 4096), (3, 4112),
         (5, 7168), (2, 8192), (2, 8208), (1, 16384), (1, 16400), (1, 65536))


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("xt,yt,wt", ((BF16, BF16, F32), (F32, BF16, BF16), (BF16, F32, F32), (F32, F32, BF16)))
@pytest.mark.parametrize("T,C", SIZES)
def test_forward(T, C, xt, yt, wt, post):
    r = rng(T, C, xt, yt, post)
    d, val, dev = inputs(r, T, C, xt, yt, wt, post)
    x, b = rows(r, T, C, xt), rows(r, T, C, yt)
    r1, n1, f1 = check_forward(d, val, dev, x, b, T, ("r", "n", "row"))
    r2, n2, f2 = check_forward(d, val, dev, x, b, T, ("r", "n", "row"))
    assert torch.equal(r1, r2) and torch.equal(n1, n2) and torch.equal(f1.codes, f2.codes) and torch.equal(f1.scales, f2.scales)
    # in place, and outputs left out
    same = x[1].clone()
    ftm.ft_block_norm(d, dev, same, b[1], T, same)
    assert torch.equal(same, r1[:T])
    only = torch.empty(T, C, dtype=TORCH[yt], device="cuda")
    ftm.ft_block_norm(d, dev, x[1], b[1], T, n=only)
    assert torch.equal(only, n1[:T])
    form = filled(T, C)
    ftm.ft_block_norm(d, dev, x[1], b[1], T, n_row=form)
    assert torch.equal(form.codes, f1.codes) and torch.equal(form.scales, f1.scales)


@pytest.mark.parametrize("T,C", ((3, 144), (2, 2064), (2, 7168)))
@pytest.mark.parametrize("left_out", (("pre",), ("gate", "token_gate"), ("post",), NAMES))
def test_weights_and_gates_left_out(T, C, left_out):
    r = rng(T, C, len(left_out))
    for post in (0, 1):
        d, val, dev = inputs(r, T, C, BF16, BF16, F32, post, left_out)
        x, b = rows(r, T, C, BF16), rows(r, T, C, BF16)
        check_forward(d, val, dev, x, b, T, ("r", "n", "row"))
        check_forward(d, val, dev, x, None, T, ("n", "row"))


def test_rows_of_zeros_and_rows_that_are_not_finite():
    T, C = 6, 1040
    r = rng(5)
    d, val, dev = inputs(r, T, C, F32, F32, F32, 1)
    xv, bv = r.normal(size=(T, C)).astype(np.float32), r.normal(size=(T, C)).astype(np.float32)
    xv[0], bv[0] = 0, 0
    xv[2, 7], bv[3, 9] = np.nan, np.inf
    rt, nt = torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda")
    form = filled(T, C)
    ftm.ft_block_norm(d, dev, cuda(xv), cuda(bv), T, rt, nt, form)
    assert not rt[0].any() and not nt[0].any() and not (form.codes[0] & 0x7F).any()
    ok = [0, 1, 4, 5]
    rv, nv = experts.norm(xv[ok].astype(float), bv[ok].astype(float), post_norm=1, eps=d["eps"], scale=d["scale"],
                          **{n: v[ok] if n == "token_gate" else v for n, v in val.items()})
    assert np.allclose(f64(rt[ok]), rv, rtol=1e-5, atol=1e-5) and np.allclose(f64(nt[ok]), nv, rtol=1e-4, atol=1e-4)
    assert torch.isnan(nt[2]).all() and torch.isnan(nt[3]).any()


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("xt,yt,wt", ((BF16, BF16, F32), (F32, BF16, BF16), (BF16, F32, F32), (F32, F32, F32)))
@pytest.mark.parametrize("T,C", SIZES + ((700, 144), (1500, 2064), (600, 4112), (520, 8208), (300, 16400)))
def test_backward(T, C, xt, yt, wt, post):
    r = rng(T, C, xt, yt, post, 2)
    d, val, dev = inputs(r, T, C, xt, yt, wt, post)
    (rv, rt), (bv, bt) = rows(r, T, C, xt), rows(r, T, C, yt)
    (drv, drt), (dnv, dnt) = tensor(r, (T, C), xt, 1e-3), tensor(r, (T, C), yt, 1e-2)
    ws = ftm.alloc_block_norm_workspace(d, T).fill_(0xFF)

    def run(block=bt, dr=drt, dn=dnt, names=NAMES):
        g = {n: torch.full(((T if n == "token_gate" else C) + 1,), 9.0, device="cuda") for n in names if n != "post" or post}
        dx = torch.full((T + 1, C), 9.0, dtype=TORCH[xt], device="cuda")
        db = None if block is None else torch.full((T + 1, C), 9.0, dtype=TORCH[yt], device="cuda")
        ftm.ft_block_norm_backward(d, dev, rt, block, dr, dn, T, dx, db, g, ws)
        return {"dx": dx, **({} if block is None else {"d_block": db}), **g}

    def check(got, block, dr, dn):
        want = experts.norm_grad(rv, block, dr, dn, post_norm=post, eps=d["eps"], scale=d["scale"], **val)
        for n, t in got.items():
            v, mag = want[n], want["mag"][n]
            kind = xt if n == "dx" else yt if n == "d_block" else F32
            sums = T if n in ("pre", "post", "gate") else 0
            err = np.abs(f64(t[:-1]) - v)
            assert np.all(err <= half(kind) * np.abs(v) + (400 + sums) * U * mag + 1e-37), (n, float((err / (mag + 1e-300)).max() / U))
            assert torch.all(t[-1] == 9.0), n

    first = run()
    check(first, bv, drv, dnv)
    again = run()
    assert all(torch.equal(first[n], again[n]) for n in first)
    zero = np.zeros_like(drv)
    check(run(dr=None), bv, zero, dnv)
    check(run(dn=None, names=("post", "gate", "token_gate")), bv, drv, zero)
    check(run(block=None, names=("pre",)), None, drv, dnv)
    # in place; some outputs left out; no workspace where no sum over the tokens is asked for
    dx, db = drt.clone(), dnt.clone()
    h = torch.empty(T, device="cuda")
    ftm.ft_block_norm_backward(d, dev, rt, bt, dx, db, T, dx, db, {"token_gate": h})
    assert torch.equal(dx, first["dx"][:T]) and torch.equal(db, first["d_block"][:T]) and torch.equal(h, first["token_gate"][:T])
    g = torch.empty(C, device="cuda")
    ftm.ft_block_norm_backward(d, dev, rt, bt, drt, dnt, T, grads={"gate": g}, ws=ws)
    assert torch.equal(g, first["gate"][:C])


def test_gradients_without_tokens_are_zeros():
    d, _, dev = inputs(rng(1), 0, 144, BF16, BF16, F32, 1)
    dev["token_gate"] = None
    g = {n: torch.full((144,), 9.0, device="cuda") for n in ("pre", "post", "gate")}
    ftm.ft_block_norm_backward(d, dev, None, None, None, None, 0, grads=g, ws=ftm.alloc_block_norm_workspace(d, 0))
    assert not any(t.any() for t in g.values())


def test_gradients_against_differences():
    """The library's own forward pass, moved by small steps, against its gradients; float32, steps of 2^-6: the
    difference's error is a third derivative's 2^-12 and float32's 2^-24 * 2^6 of sums of some hundred."""
    T, C = 3, 48
    r = rng(77)
    d, val, dev = inputs(r, T, C, F32, F32, F32, 1)
    x, b = (cuda(r.normal(size=(T, C)).astype(np.float32)) for _ in range(2))
    dr, dn = (cuda(r.normal(size=(T, C)).astype(np.float32)) for _ in range(2))

    def outs(x=x, b=b, **kw):
        rt, nt = torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda")
        ftm.ft_block_norm(d, {**dev, **kw}, x, b, T, rt, nt)
        return rt, nt

    rt, _ = outs()
    dx, db = torch.empty(T, C, device="cuda"), torch.empty(T, C, device="cuda")
    g = {n: torch.empty_like(dev[n]) for n in NAMES}
    ftm.ft_block_norm_backward(d, dev, rt, b, dr, dn, T, dx, db, g, ftm.alloc_block_norm_workspace(d, T))
    h = 2.0 ** -6
    for name, at, grad in (("x", x, dx), ("b", b, db)) + tuple((n, dev[n], g[n]) for n in NAMES):
        for i in r.choice(at.numel(), min(12, at.numel()), replace=False):
            up, down = at.clone(), at.clone()
            up.view(-1)[i] += h
            down.view(-1)[i] -= h
            f = [(f64(a) * f64(dr)).sum() + (f64(n) * f64(dn)).sum() for a, n in (outs(**{name: up}), outs(**{name: down}))]
            assert abs((f[0] - f[1]) / (2 * h) - float(grad.view(-1)[i])) < 2e-2, (name, i)
