"""The norms before and after a block: rows that are not finite at any channel, the least values that a norm without eps is
defined for, and more rows than run at once, a part of a round past the last whole one.  Against the 64-bit oracle, with the tolerances of
tests/test_gpu_norm.py."""
import numpy as np
import pytest
import torch

import paper_2608_16157_amd as ftm
from oracle import experts
from tests.test_gpu_dense import BF16, F32, TORCH, cuda, f64, filled, rng
from tests.test_gpu_norm import NAMES, U, check_forward, forward_tolerance, half, inputs, rows, tensor

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("kind", (BF16, F32))
@pytest.mark.parametrize("C", (16, 48, 512, 528, 1040, 2064, 7168, 8192, 8208, 16400))
def test_infinities_at_any_channel(C, kind, post):
    """An infinity leaves the other channels of its row what the definition says, at the first channel as at the last, which
    the threads past the end of a row read as well: of r those of x, of n zeros; a NaN from the block makes its row's n NaN."""
    places = [(c, v) for c in sorted({0, C // 2, C - 8, C - 2, C - 1}) for v in (np.inf, -np.inf)]
    T = 2 * len(places) + 1
    r = rng(C, kind, post, 41)
    d, val, dev = inputs(r, T, C, kind, kind, F32, post)
    (xv, x), (bv, b) = rows(r, T, C, kind), rows(r, T, C, kind)
    for i, (c, v) in enumerate(places):
        x[2 * i, c] = xv[2 * i, c] = v
        b[2 * i + 1, c] = bv[2 * i + 1, c] = v
    form = filled(T, C)
    rt, nt = torch.empty_like(x), torch.empty_like(x)
    ftm.ft_block_norm(d, dev, x, b, T, rt, nt, form)
    with np.errstate(invalid="ignore"):
        rv, nv = experts.norm(xv, bv, post_norm=post, eps=d["eps"], scale=d["scale"], **val)
        step = forward_tolerance(d, val, xv, bv)
    fin = np.isfinite(rv).all(axis=1, keepdims=True)
    step = np.where(np.isfinite(step), step, 0)
    mag = np.where(np.isfinite(xv), np.abs(xv), 0) + step
    rms = np.where(fin, experts._rms(np.where(fin, rv, 0), d["eps"]), np.inf)
    back = 1 + np.sqrt((mag ** 2).mean(axis=1, keepdims=True)) / rms
    for got, want, tol in ((f64(rt), rv, 61 * U * (step + np.abs(rv))), (f64(nt), nv, 121 * U * np.abs(val["pre"]) * mag / rms * back)):
        assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(np.isinf(got), np.isinf(want))
        ok = np.isfinite(want)
        assert np.all(np.abs(got[ok] - want[ok]) <= half(kind) * np.abs(want[ok]) + tol[ok])
    codes = form.codes[:, :C].cpu().numpy()
    assert np.array_equal((codes & 0x7F) == 0x7F, ~np.isfinite(nv))
    zero = np.isfinite(nv) & (nv == 0)
    assert zero.any() and not (codes[zero] & 0x7F).any()


def check_backward(d, val, dev, r, b, dr, dn, T):
    """Every gradient; r, b, dr, dn: (values, tensor)."""
    got = {n: torch.full((T if n == "token_gate" else d["channels"],), 9.0, device="cuda") for n in NAMES if n != "post" or d["post_norm"]}
    grads = dict(got)
    got["dx"], got["d_block"] = torch.empty_like(r[1]), torch.empty_like(b[1])
    ws = ftm.alloc_block_norm_workspace(d, T).fill_(0xFF)
    ftm.ft_block_norm_backward(d, dev, r[1], b[1], dr[1], dn[1], T, got["dx"], got["d_block"], grads, ws)
    want = experts.norm_grad(r[0], b[0], dr[0], dn[0], post_norm=d["post_norm"], eps=d["eps"], scale=d["scale"], **val)
    for n, t in got.items():
        err, v, mag = np.abs(f64(t) - want[n]), want[n], want["mag"][n]
        kind = d["x_dtype"] if n == "dx" else d["y_dtype"] if n == "d_block" else F32
        sums = T if n in ("pre", "post", "gate") else 0
        assert np.all(err <= half(kind) * np.abs(v) + (400 + sums) * U * mag + 1e-37), n
    return got


def least(r, T, C, kind):
    """Values of either sign from 2^-63 to 2^-61."""
    t = cuda(r.uniform(2.0 ** -63, 2.0 ** -61, (T, C)) * r.choice((-1.0, 1.0), (T, C))).to(TORCH[kind])
    return f64(t), t


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("kind", (BF16, F32))
@pytest.mark.parametrize("C", (16, 144, 1040, 7168, 8208, 16400))
def test_least_rows_without_eps(C, kind, post):
    """Single squares may be subnormal: each of up to 88 additions is off by 2^-150 more, 5.5 u of a sum of 16 2^-126 and
    more, and 1/rms by half of it: inside the 50 u of the tolerances.  Gradients with one of the two rows at the bound, and with both."""
    T = 5
    r = rng(C, kind, post, 42)
    d, val, dev = inputs(r, T, C, kind, kind, F32, post)
    d["eps"] = 0.0
    small, normal = least(r, T, C, kind), rows(r, T, C, kind)
    check_forward(d, val, dev, small, None, T, ("n", "row"))
    check_forward(d, val, dev, normal, small, T, ("r", "n", "row"))
    for (rv, rt), (bv, bt) in ((small, normal), (normal, small), (small, least(r, T, C, kind))):
        (drv, drt), (dnv, dnt) = tensor(r, (T, C), kind, 2.0 ** -10), tensor(r, (T, C), kind, 2.0 ** -10)
        check_backward(d, val, dev, (rv, rt), (bv, bt), (drv, drt), (dnv, dnt), T)


TYPES = ((BF16, BF16, F32), (F32, BF16, BF16), (BF16, F32, F32), (F32, F32, BF16))


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("xt,yt,wt", TYPES)
@pytest.mark.parametrize("T,C", ((6200, 144), (6147, 16), (1600, 1040), (800, 2064), (300, 7168), (300, 8208), (290, 16400)))
def test_forward_of_more_rows_than_run_at_once(T, C, xt, yt, wt, post):
    """A workgroup takes several rows, each requested while the one before is on the way: rows of sizes from 10^-2 to 10^2 and gates
    of their own would show a row, its gate or its sums in the place of another's."""
    r = rng(T, C, xt, yt, post, 43)
    d, val, dev = inputs(r, T, C, xt, yt, wt, post)
    x, b = rows(r, T, C, xt), rows(r, T, C, yt)
    r1, n1, _ = check_forward(d, val, dev, x, b, T, ("r", "n", "row"))
    check_forward(d, val, dev, x, None, T, ("n",))
    same, n2 = x[1].clone(), torch.empty_like(b[1])
    ftm.ft_block_norm(d, dev, same, b[1], T, same, n2)      # in place
    assert torch.equal(same, r1[:T]) and torch.equal(n2, n1[:T])


@pytest.mark.parametrize("post", (0, 1))
@pytest.mark.parametrize("xt,yt,wt", TYPES)
@pytest.mark.parametrize("T,C", ((4200, 144), (4200, 512), (4099, 16), (1100, 528), (1100, 2048), (600, 4096), (300, 7168), (300, 16384)))
def test_backward_of_more_rows_than_run_at_once(T, C, xt, yt, wt, post):
    r = rng(T, C, xt, yt, post, 44)
    d, val, dev = inputs(r, T, C, xt, yt, wt, post)
    rr, b, dr, dn = rows(r, T, C, xt), rows(r, T, C, yt), tensor(r, (T, C), xt, 1e-3), tensor(r, (T, C), yt, 1e-2)
    got = check_backward(d, val, dev, rr, b, dr, dn, T)
    dx, db, h = dr[1].clone(), dn[1].clone(), torch.empty(T, device="cuda")
    ftm.ft_block_norm_backward(d, dev, rr[1], b[1], dx, db, T, dx, db, {"token_gate": h})      # in place
    assert torch.equal(dx, got["dx"]) and torch.equal(db, got["d_block"]) and torch.equal(h, got["token_gate"])
