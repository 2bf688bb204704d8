"""Weight gradients of the experts in tiles of 256 x 256 with the next run of experts' columns read ahead, which takes enough whole
tiles (128 to 224, or 768 and more, three quarters of them results) and 16 experts: unlike groups in several runs, reductions of
more blocks than the tile's rings hold, runs without any row, a partial last run, last tiles narrower than 256.  Against the
64-bit oracle, with the tolerance of the other products."""
import numpy as np
import pytest
import torch

import paper_2608_16157_amd as ftm
from oracle import experts
from tests.test_gpu_dense import BF16, F32, TORCH, assert_product, cuda, form_of, matrix, rng
from tests.test_gpu_experts import tables_of

pytestmark = pytest.mark.gpu


def large_tiles(E, N, K):
    tiles = E * -(-N // 256) * -(-K // 256)
    return (tiles >= 768 or 128 < tiles <= 224) and 4 * E * N * K >= 3 * 65536 * tiles


def groups(sizes, align=128):
    """Tables of groups of the given sizes, from a routing of one expert per token."""
    r = rng(len(sizes), 51)
    ids = r.permutation(np.repeat(np.arange(len(sizes)), sizes)).astype(np.int32)[:, None]
    rows = max(align, int(sum(-(-n // align) * align for n in sizes)) + align)       # and some behind the last group
    return {"n_experts": len(sizes), "top_k": 1, "align": align, "rows": rows}, experts.sort(ids, 0, len(sizes), align, rows), len(ids)


EVEN = (140, 0, 1300, 128, 700, 1, 260, 90)
CASES = ((EVEN + (0,) * 8 + (900, 5), 768, 768),                       # 18 experts, the second run empty
         ((0, 129, 640, 0, 385, 1025, 3, 0) + EVEN + (770, 0, 130, 1), 1008, 512),      # 20
         ((0,) * 8 + EVEN + (0, 0, 0, 900), 512, 1008),                # the first run empty, the last one partial
         (EVEN + (0,) * 16 + EVEN[::-1], 512, 752),                    # 32, two empty runs between
         ((64,) * 95 + (1100, 0, 900), 768, 592))                      # 98 experts, 882 tiles; 13 runs


@pytest.mark.parametrize("sizes,N,K", CASES)
def test_large_tiles_of_runs_of_experts(sizes, N, K):
    E = len(sizes)
    assert E >= 16 and large_tiles(E, N, K)
    d, want, T = groups(sizes)
    s, end = tables_of(want), int(want["off"][-1])
    r = rng(E, N, K, 52)
    real = np.zeros((d["rows"], 1))
    real[:end, 0] = want["row_pair"][:end] >= 0
    (dc, a), (xc, b) = (form_of((matrix(r, d["rows"], C, spread=1)[0] * real).T) for C in (N, K))
    dc.codes[:, end:], xc.codes[:, end:] = 0x7F, 0x7F                  # behind the last group: not read
    v, mag = experts.weight_grad(want, a.T, b.T)
    for kind, kw in ((BF16, {}), (F32, {}), (F32, {"accumulate": True})):
        dw = torch.full((E + 1, N, K), 3.0, dtype=TORCH[kind], device="cuda")
        ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, dw, **kw)
        assert torch.all(dw[E] == 3.0)
        if kw:
            assert torch.all(dw[:E][cuda(want["count"] == 0)] == 3.0)
            # two roundings of sums with the 3, beyond those of the product
            err = np.abs(dw[:E].double().cpu().numpy() - 3.0 - v)
            assert np.all(err <= (max(sizes) + max(sizes) // 128 + 4) * 2.0 ** -24 * (mag + 3.0))
        else:
            assert_product(dw[:E], v, mag, max(sizes), kind)
            assert not dw[:E][cuda(want["count"] == 0)].any()
        again = torch.full_like(dw, 3.0)
        ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, again, **kw)
        assert torch.equal(dw, again)
