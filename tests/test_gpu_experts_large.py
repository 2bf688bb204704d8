"""The routed experts in training and the norms on buffers past 4 GiB, the largest sizes, against the same calls on small
copies of the ends.  The tolerances are those of the small tests; most results have to be equal."""
import numpy as np
import pytest
import torch

import paper_2608_16157_amd as ftm
from tests.test_gpu_dense import ACT, BF16, F32
from tests.test_gpu_experts import desc

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def give_back():
    yield
    torch.cuda.empty_cache()


def tables(d, ids, T):
    s = ftm.SortBuffers(d, T)
    ftm.ft_expert_sort(d, ids, T, s, ftm.alloc_sort_workspace(d, T))
    return s


def test_rows_past_4_gib():
    """All rows of 2^20: tokens' rows and their 8-bit forms, back to the tokens, the gates' gradients."""
    T, E, k, C = 131072, 8, 8, 2064
    d = {"n_experts": E, "top_k": k, "align": 128, "rows": 1 << 20}
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.argsort(torch.rand(T, E, generator=g, device="cuda"), dim=1)[:, :k].to(torch.int32).contiguous()
    ids[-1, -1] = -1
    s = tables(d, ids, T)
    assert int(s.off[E]) == 1 << 20 and int(s.dropped) == 0 and int(s.pair_row[-1, -1]) == -1
    x = torch.randn(T, C, generator=g, device="cuda")
    rows = torch.empty(1 << 20, C, device="cuda")                      # 8.7 GB
    row, col = ftm.ActCodes(1 << 20, C), ftm.ActCodes(C, 1 << 20)
    ftm.ft_expert_gather(d, s, x, T, C, rows=rows, row=row, col=col)
    back = torch.empty(T, C, device="cuda")
    ftm.ft_expert_combine(d, s, rows, T, C, back)
    d_w = torch.empty(T, k, device="cuda")
    ftm.ft_expert_gate_grad(d, s, rows, x, T, C, d_w)
    for t in (0, 65535, T - 2, T - 1):
        want = 8 if t < T - 1 else 7
        assert torch.allclose(back[t], want * x[t], rtol=1e-6)
        assert torch.allclose(d_w[t, :want], (x[t].double() ** 2).sum().float().expand(want), rtol=C * 2.0 ** -24)
    assert float(d_w[-1, -1]) == 0
    # the last 128 rows' forms, from a call of their own
    p = s.row_pair[-128:].long()
    end = torch.where((p >= 0)[:, None], x[p.clamp(min=0) // k], torch.zeros(1, device="cuda"))
    assert torch.equal(rows[-128:], end)
    r2, c2 = ftm.ActCodes(128, C), ftm.ActCodes(C, 128)
    ftm.ft_act_quantize(end, 128, C, r2, c2)
    assert torch.equal(row.codes[-128:], r2.codes) and torch.equal(row.scales[:, -128:], r2.scales)
    assert torch.equal(col.codes[:, -128:], c2.codes) and torch.equal(col.scales[-1:, :C], c2.scales[:, :C])


def test_weights_and_gradients_past_4_gib():
    n, N, K, T = 66, 8208, 8192, 300
    d = desc(n, 1, 128, T)
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.full((T, 1), n - 1, dtype=torch.int32, device="cuda")
    ids[:40] = n - 2
    s = tables(d, ids, T)
    R = d["rows"]
    w = {"w": torch.zeros(n, N, K, dtype=torch.uint8, device="cuda"), "s": torch.ones(n, 65, 64, device="cuda")}   # 4.4 GB
    w["w"][-2:] = torch.randint(0, 120, (2, N, K), generator=g, device="cuda", dtype=torch.uint8)
    x = (torch.randn(T, K, generator=g, device="cuda")).to(torch.bfloat16)
    xr, xc = ftm.ActCodes(R, K), ftm.ActCodes(K, R)
    ftm.ft_expert_gather(d, s, x, T, K, row=xr, col=xc)
    lin = {"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": BF16}
    y = torch.empty(R, N, dtype=torch.bfloat16, device="cuda")
    ftm.ft_expert_linear(d, lin, w, xr, s, T, y)
    for e, tokens in ((n - 2, slice(0, 40)), (n - 1, slice(40, T))):
        m = tokens.stop - tokens.start
        one = torch.empty(m, N, dtype=torch.bfloat16, device="cuda")
        ftm.ft_linear({**lin, "x_dtype": BF16}, {"w": w["w"][e], "s": w["s"][e]}, x[tokens].contiguous(), m, one,
                      ftm.alloc_linear_workspace({**lin, "x_dtype": BF16}, m))
        o = int(s.off[e])
        # sums in another order (a split reduction): float32's rounding, then bf16's
        assert (y[o:o + m].float() - one.float()).norm() <= 2.0 ** -8 * one.float().norm()
    wt = {"w": torch.empty(n, K, 8320, dtype=torch.uint8, device="cuda"), "s": torch.empty(n, 64, 65, device="cuda")}
    ftm.ft_expert_linear_transpose(n, N, K, w, wt)
    assert torch.equal(wt["w"][-1, :, :N], w["w"][-1].t()) and torch.equal(wt["s"][-1], w["s"][-1].t())
    del w, wt
    dyc = ftm.ActCodes(N, R)
    ftm.ft_expert_gather(d, s, y[:T].contiguous(), T, N, col=dyc)
    for kind, dt in ((torch.bfloat16, BF16), (torch.float32, F32)):
        dw = torch.full((n, N, K), 3.0, dtype=kind, device="cuda")      # 8.9 and 17.8 GB
        ftm.ft_expert_weight_grad(d, N, K, dyc, xc, s, T, dw)
        assert not dw[:n - 2].any()
        for e, tokens in ((n - 2, slice(0, 40)), (n - 1, slice(40, T))):
            m = tokens.stop - tokens.start
            a, b = ftm.ActCodes(N, m), ftm.ActCodes(K, m)
            ftm.ft_act_quantize(y[:T][tokens].contiguous(), m, N, col=a)
            ftm.ft_act_quantize(x[tokens].contiguous(), m, K, col=b)
            one = torch.empty(N, K, dtype=kind, device="cuda")
            ftm.ft_linear_weight_grad(N, K, m, a, b, one)
            assert torch.equal(dw[e], one)
        del dw


def test_norms_past_4_gib():
    T, C = 70001, 32784
    d = {"channels": C, "x_dtype": BF16, "y_dtype": BF16, "w_dtype": F32, "post_norm": 1, "eps": 1e-6, "scale": 0.5}
    g = torch.Generator(device="cuda").manual_seed(3)
    new = lambda: torch.randn(T, C, generator=g, device="cuda", dtype=torch.bfloat16)      # 4.6 GB each
    x, b, dr, dn = new(), new(), new(), new()
    params = {"pre": torch.rand(C, device="cuda"), "post": torch.rand(C, device="cuda"), "gate": torch.rand(C, device="cuda"),
              "token_gate": torch.rand(T, device="cuda")}
    r, n, form = torch.empty_like(x), torch.empty_like(x), ftm.ActCodes(T, C)
    ftm.ft_block_norm(d, params, x, b, T, r, n, form)
    dx, db, h = torch.empty_like(x), torch.empty_like(x), torch.empty(T, device="cuda")
    ftm.ft_block_norm_backward(d, params, r, b, dr, dn, T, dx, db, {"token_gate": h})
    few = 3
    end = {**params, "token_gate": params["token_gate"][-few:].contiguous()}
    cut = lambda t: t[-few:].contiguous()
    r2, n2, f2 = (torch.empty(few, C, dtype=torch.bfloat16, device="cuda") for _ in range(2)), None, ftm.ActCodes(few, C)
    r2, n2 = r2
    ftm.ft_block_norm(d, end, cut(x), cut(b), few, r2, n2, f2)
    assert torch.equal(r[-few:], r2) and torch.equal(n[-few:], n2) and torch.equal(form.codes[-few:], f2.codes)
    assert torch.equal(form.scales[:, T - few:T], f2.scales[:, :few]) and torch.all(form.scales[:, T:] == 127)
    dx2, db2, h2 = torch.empty_like(r2), torch.empty_like(r2), torch.empty(few, device="cuda")
    ftm.ft_block_norm_backward(d, end, cut(r), cut(b), cut(dr), cut(dn), few, dx2, db2, {"token_gate": h2})
    assert torch.equal(dx[-few:], dx2) and torch.equal(db[-few:], db2) and torch.equal(h[-few:], h2)


def test_a_million_tokens():
    """The most tokens: tables, rows of a few, norm and column sums."""
    T, C = 1 << 20, 16
    d = {"n_experts": 1024, "top_k": 1, "first": 1000, "local": 24, "align": 16, "rows": 1 << 19}
    ids = (torch.arange(T, device="cuda", dtype=torch.int32) % 1024)[:, None].contiguous()
    s = tables(d, ids, T)
    assert torch.all(s.count == 1024) and int(s.off[24]) == 24 * 1024
    x = torch.arange(T, device="cuda", dtype=torch.float32)[:, None].expand(T, C).contiguous()
    rows = torch.zeros(1 << 19, C, device="cuda")
    ftm.ft_expert_gather(d, s, x, T, C, rows=rows)
    want = (torch.arange(24, device="cuda")[:, None] + 1000 + 1024 * torch.arange(1024, device="cuda")[None]).view(-1)
    assert torch.equal(rows[:24 * 1024, 3].long(), want) and not rows[24 * 1024:].any()
    back = torch.empty(T, C, device="cuda")
    ftm.ft_expert_combine(d, s, rows, T, C, back)
    assert torch.equal(back, torch.where(ids >= 1000, x, torch.zeros(1, device="cuda")))
    nd = {"channels": C, "x_dtype": F32, "y_dtype": F32, "w_dtype": F32, "eps": 0.0, "scale": 1.0}
    one = torch.ones(T, C, device="cuda")
    dx, pre, gate = torch.empty(T, C, device="cuda"), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    ftm.ft_block_norm_backward(nd, {}, one, one, one, one, T, dx, None, {"pre": pre, "gate": gate}, ftm.alloc_block_norm_workspace(nd, T))
    # ones everywhere: n = 1, the norm takes its own gradient away; whole numbers below 2^24
    assert torch.equal(dx, one) and torch.all(pre == T) and torch.all(gate == T)


def test_combine_of_the_most_channels():
    """More blocks than one dimension of a grid holds: 2^20 tokens of 20480 channels, 43 GB of results."""
    T, C = 1 << 20, 20480
    d = {"n_experts": 4, "top_k": 1, "align": 16, "rows": 16}
    s = ftm.SortBuffers(d, T)
    s.pair_row.fill_(-1)
    for t, row in ((0, 3), (T // 2, 7), (T - 1, 15)):
        s.pair_row[t, 0] = row
    rows = torch.arange(16, device="cuda", dtype=torch.float32)[:, None].expand(16, C).to(torch.bfloat16).contiguous()
    y = torch.full((T, C), 9.0, dtype=torch.bfloat16, device="cuda")
    ftm.ft_expert_combine(d, s, rows, T, C, y)
    for t, row in ((0, 3), (T // 2, 7), (T - 1, 15)):
        assert torch.all(y[t] == row)
        y[t] = 0
    assert all(not part.any() for part in y.split(1 << 17))
