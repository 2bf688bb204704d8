"""The norms before and after a block: rows that are not finite at any channel, and the least values that a norm without eps is
defined for.  Against the 64-bit oracle, with the tolerances of
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
        got = {n: torch.empty(T if n == "token_gate" else C, device="cuda") for n in NAMES if n != "post" or post}
        grads = dict(got)
        got["dx"], got["d_block"] = torch.empty_like(rt), torch.empty_like(bt)
        ftm.ft_block_norm_backward(d, dev, rt, bt, drt, dnt, T, got["dx"], got["d_block"], grads, ftm.alloc_block_norm_workspace(d, T))
        want = experts.norm_grad(rv, bv, drv, dnv, post_norm=post, eps=0.0, scale=d["scale"], **val)
        for n, t in got.items():
            err, v, mag = np.abs(f64(t) - want[n]), want[n], want["mag"][n]
            to = kind if n in ("dx", "d_block") else F32
            assert np.all(err <= half(to) * np.abs(v) + (400 + T) * U * mag), n
