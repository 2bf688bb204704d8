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
