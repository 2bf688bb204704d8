"""The norms before and after a block: rows that are not finite at any channel.  Against the 64-bit oracle, with the tolerances of
tests/test_gpu_norm.py."""
import numpy as np
import pytest
import torch

import paper_2608_16157_amd as ftm
from oracle import experts
from tests.test_gpu_dense import BF16, F32, TORCH, cuda, f64, filled, rng
from tests.test_gpu_norm import U, forward_tolerance, half, inputs, rows

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
