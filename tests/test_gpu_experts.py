"""The routed experts in training on the GPU against the 64-bit oracle: pairs sorted by expert, rows of tokens in that
order and back, products over the groups and their gradients.

Tolerances, from the arithmetic (u = 2^-24; a rounding to bf16 is 2^-8 of the value):
* tables are whole numbers and equal;
* rows without weights are copies (or the exact 8-bit form of what was given); with weights one float32 product is
  rounded, and the oracle's rows are rounded the same way before they are compared;
* combine: each of up to k fused multiply-adds rounds a partial sum, which the sum of magnitudes bounds: k u of it;
* gates' gradients: C products in chains of at most C / 256 + 8, six sums across the lanes, three across the waves; C u of
  the sum of magnitudes holds for C of 64 and more, 24 u below;
* products: as the dense ones (assert_product).
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_16157_amd as ftm
from oracle import dense, experts
from tests.test_gpu_dense import (ACT, BF16, F32, TORCH, assert_exact_form, assert_product, cuda, f64, filled, form_of, matrix, rng,
                                  weight)

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def desc(E, k, align, T, first=0, local=None, rows=None):
    d = {"n_experts": E, "top_k": k, "first": first, "local": E if local is None else local, "align": align}
    d["rows"] = ftm.ft_expert_sort_rows(d, T) if rows is None else rows
    assert d["rows"] > 0
    return d


def routing(r, T, E, k, skew=1.0):
    """Distinct experts per token, the first ones more often."""
    key = r.gumbel(size=(T, E)) - skew * np.log(1.0 + np.arange(E))
    return np.ascontiguousarray(np.argsort(-key, axis=1)[:, :k]).astype(np.int32)


def quantize(v):
    """dense.quantize, also of no rows or no columns."""
    if v.size:
        return dense.quantize(v)
    return np.zeros((len(v), dense.pad128(v.shape[1])), np.uint8), np.zeros((dense.pad128(v.shape[1]) // 128, len(v)), np.uint8)


def run_sort(d, ids, mask=None):
    T = ids.shape[0]
    s = ftm.SortBuffers(d, T)
    for n in ("row_pair", "pair_row", "off", "count", "dropped"):
        getattr(s, n).fill_(-77)
    ws = ftm.alloc_sort_workspace(d, T).fill_(0xA5)
    ftm.ft_expert_sort(d, cuda(ids), T, s, ws, mask=None if mask is None else cuda(mask))
    return s


def assert_tables(s, d, ids, mask=None):
    want = experts.sort(ids, d["first"], d["local"], d["align"], d["rows"], mask)
    for n in ("row_pair", "pair_row", "off", "count", "dropped"):
        assert np.array_equal(getattr(s, n).cpu().numpy(), want[n]), n
    return want


def tables_of(want):
    """Device tables of the oracle's."""
    c = lambda n: cuda(want[n].astype(np.int32))
    return ftm.SortBuffers.of(c("row_pair"), c("pair_row"), c("off"), c("count"), c("dropped"))


# ----------------------------------------------------------------------------------------- tables

@pytest.mark.parametrize("align", (16, 128))
@pytest.mark.parametrize("T,E,k,first,local", ((1, 1, 1, 0, 1), (1, 8, 2, 0, 8), (3, 5, 5, 0, 5), (17, 64, 8, 16, 8), (63, 128, 8, 0, 128),
                                               (130, 60, 4, 59, 1), (511, 256, 8, 0, 256), (200, 1024, 64, 0, 1024),
                                               (513, 384, 8, 100, 65)))
def test_tables(T, E, k, first, local, align):
    r = rng(T, E, k, align)
    ids = routing(r, T, E, k)
    d = desc(E, k, align, T, first, local)
    assert_tables(run_sort(d, ids), d, ids)
    mask = (r.random(T) < 0.7).astype(np.uint8)
    assert_tables(run_sort(d, ids, mask), d, ids, mask)
    assert_tables(run_sort(d, ids, np.zeros(T, np.uint8)), d, ids, np.zeros(T, np.uint8))


@pytest.mark.parametrize("T,E,k", ((4097, 7, 1), (1025, 32, 4), (3000, 1024, 3), (20000, 12, 2)))
def test_tables_over_several_workgroups(T, E, k):
    r = rng(T, E, k, 5)
    ids = routing(r, T, E, k)
    d = desc(E, k, 16, T)
    s = run_sort(d, ids)
    # the oracle of so many pairs, expert by expert
    flat = ids.reshape(-1)
    at = 0
    row_pair = np.full(d["rows"], -1)
    for e in range(E):
        p = np.nonzero(flat == e)[0]
        assert int(s.off[e]) == at and int(s.count[e]) == len(p)
        row_pair[at:at + len(p)] = p
        at += -(-len(p) // 16) * 16
    assert int(s.off[E]) == at and int(s.dropped) == 0
    assert np.array_equal(s.row_pair.cpu().numpy(), row_pair)
    rows = np.nonzero(row_pair >= 0)[0]
    pair_row = np.empty(T * k, int)
    pair_row[row_pair[rows]] = rows
    assert np.array_equal(s.pair_row.cpu().numpy().reshape(-1), pair_row)
    assert torch.equal(s.row_pair, run_sort(d, ids).row_pair)


def test_tables_of_more_pairs_than_one_round_of_workgroups_holds():
    """2^23 pairs: every workgroup places several times what it holds at once.  Most find no place."""
    T, E, k = 1 << 20, 16, 8
    d = {"n_experts": E, "top_k": k, "align": 16, "rows": 1 << 20}
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = torch.randint(-2, E + 2, (T, k), generator=g, device="cuda", dtype=torch.int32)
    s, ws = ftm.SortBuffers(d, T), ftm.alloc_sort_workspace(d, T)
    ftm.ft_expert_sort(d, ids, T, s, ws)
    flat = ids.view(-1).cpu().numpy()
    at, lost = 0, 0
    row_pair, pair_row = np.full(1 << 20, -1), np.full(T * k, -1)
    for e in range(E):
        p = np.nonzero(flat == e)[0]
        got = p[:(1 << 20) - at]
        row_pair[at:at + len(got)], pair_row[got] = got, at + np.arange(len(got))
        assert int(s.off[e]) == at and int(s.count[e]) == len(got)
        lost += len(p) - len(got)
        at = min(1 << 20, at + -(-len(p) // 16) * 16)
    assert int(s.off[E]) == at == 1 << 20 and int(s.dropped) == lost
    assert np.array_equal(s.row_pair.cpu().numpy(), row_pair) and np.array_equal(s.pair_row.cpu().numpy().reshape(-1), pair_row)


@pytest.mark.parametrize("align,rows", ((16, 16), (16, 48), (16, 160), (128, 128), (128, 384)))
def test_pairs_without_a_place(align, rows):
    r = rng(align, rows)
    ids = routing(r, 60, 6, 3)
    d = desc(6, 3, align, 60, rows=rows)
    want = assert_tables(run_sort(d, ids), d, ids)
    assert want["dropped"][0] > 0


def test_ids_that_are_no_experts_and_the_same_expert_twice():
    ids = np.array([[3, 3], [-1, 2], [1 << 30, 3], [-(1 << 31), 4], [3, 5], [2, 2]], np.int32)
    for first, local in ((0, 5), (2, 2), (3, 1)):
        d = desc(5, 2, 16, 6, first, local)
        assert_tables(run_sort(d, ids), d, ids)


def test_tables_without_tokens():
    d = desc(5, 2, 128, 0, rows=256)
    s = ftm.SortBuffers(d, 0)
    for n in ("row_pair", "off", "count", "dropped"):
        getattr(s, n).fill_(9)
    ftm.ft_expert_sort(d, torch.empty(0, 2, dtype=torch.int32, device="cuda"), 0, s, ftm.alloc_sort_workspace(d, 0))
    assert torch.all(s.row_pair == -1) and not s.off.any() and not s.count.any() and not s.dropped.any()


# ------------------------------------------------------------------------------------------- rows

ROWS = ((1, 1, 1, 16), (3, 8, 2, 48), (17, 16, 4, 144), (40, 8, 8, 528), (130, 60, 6, 256), (33, 64, 33, 1040), (5, 4, 2, 2064))   # T, E, k, C


def layout(r, T, E, k, align, part=False):
    """A routing with masked tokens, its oracle tables and device tables."""
    d = desc(E, k, align, T, E // 4 if part else 0, max(1, E // 2) if part else E)
    mask = (r.random(T) < 0.8).astype(np.uint8)
    ids = routing(r, T, E, k)
    want = experts.sort(ids, d["first"], d["local"], align, d["rows"], mask)
    return d, want, tables_of(want)


@pytest.mark.parametrize("part", (False, True))
@pytest.mark.parametrize("xt,ot", ((BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)))
@pytest.mark.parametrize("T,E,k,C", ROWS)
def test_gather_of_plain_rows(T, E, k, C, xt, ot, part):
    r = rng(T, E, C, xt, ot)
    d, want, s = layout(r, T, E, k, 16, part)
    xv, x = matrix(r, T, C, xt)
    w = r.normal(size=(T, k)).astype(np.float32)
    end = want["off"][-1]
    for weights in (None, w):
        out = torch.full((d["rows"], C), 7.0, dtype=TORCH[ot], device="cuda")
        ftm.ft_expert_gather(d, s, x, T, C, weights=None if weights is None else cuda(weights), rows=out)
        v = experts.gather(want, xv, weights).astype(np.float32)     # one float32 rounding of an exact product
        assert torch.equal(out[:end], cuda(v).to(TORCH[ot])) and torch.all(out[end:] == 7.0)


def assert_behind(form, rows_end, row):
    """What lies behind the last group is as filled() left it."""
    if row:
        assert torch.all(form.codes[rows_end:] == 0xA5) and torch.all(form.scales[:, rows_end:] == 0x5A)
    else:
        assert torch.all(form.codes[:, rows_end:] == 0xA5) and torch.all(form.scales[rows_end // 128:] == 0x5A)


@pytest.mark.parametrize("xt", (BF16, F32))
@pytest.mark.parametrize("align", (16, 128))
@pytest.mark.parametrize("T,E,k,C", ROWS)
def test_gather_in_8_bits(T, E, k, C, align, xt):
    r = rng(T, E, C, align, xt, 1)
    d, want, s = layout(r, T, E, k, align)
    xv, x = matrix(r, T, C, xt, spread=8)
    w = r.normal(size=(T, k)).astype(np.float32)
    end = int(want["off"][-1])
    for weights in (None, w):
        arg = {} if weights is None else {"weights": cuda(weights)}
        v = experts.gather(want, xv, weights)
        if weights is not None:
            v = v.astype(np.float32).astype(np.float64)
        row = filled(d["rows"], C)
        ftm.ft_expert_gather(d, s, x, T, C, row=row, **arg)
        codes, scales = quantize(v)
        assert np.array_equal(row.codes[:end].cpu().numpy(), codes) and np.array_equal(row.scales[:, :end].cpu().numpy(), scales)
        assert_behind(row, end, True)
        if align != 128:
            continue
        both, col, only = filled(d["rows"], C), filled(C, d["rows"]), filled(C, d["rows"])
        plain = torch.full((d["rows"], C), 7.0, device="cuda")
        ftm.ft_expert_gather(d, s, x, T, C, row=both, col=col, rows=plain, **arg)
        ftm.ft_expert_gather(d, s, x, T, C, col=only, **arg)
        assert torch.equal(both.codes, row.codes) and torch.equal(both.scales[:, :end], row.scales[:, :end])
        codes, scales = quantize(v.T)
        assert np.array_equal(col.codes[:, :end].cpu().numpy(), codes[:, :end])
        assert np.array_equal(col.scales[:end // 128, :C].cpu().numpy(), scales)
        assert_behind(col, end, False)
        assert torch.equal(col.codes, only.codes) and torch.equal(col.scales, only.scales)
        assert np.array_equal(f64(plain[:end]), v.astype(np.float32)) and torch.all(plain[end:] == 7.0)


def test_rows_that_are_not_finite():
    """Values that are not finite stay in their rows: padding is zeros, and other rows' blocks keep their scales."""
    T, E, k, C = 5, 3, 2, 256
    r = rng(3)
    d, want, s = layout(r, T, E, k, 128)
    x = r.normal(size=(T, C)).astype(np.float32)
    x[1, 3], x[2], x[3, 130] = np.nan, np.inf, -np.inf
    row, col = filled(d["rows"], C), filled(C, d["rows"])
    ftm.ft_expert_gather(d, s, cuda(x), T, C, row=row, col=col)
    v = np.zeros((want["off"][-1], C))
    for i, p in enumerate(want["row_pair"][:len(v)]):
        if p >= 0:
            v[i] = x[p // k]
    end = len(v)
    for form, m in ((row, v), (col, v.T)):
        with np.errstate(invalid="ignore"):
            codes, scales = quantize(m)
        got = form.codes[:end] if form is row else form.codes[:, :end]
        bad = ~np.isfinite(m)
        got = got.cpu().numpy()
        assert np.all((got[bad] & 0x7F) == 0x7F) and np.array_equal(got[~bad], codes[:, :m.shape[1]][~bad])
        want_scales = scales if form is row else scales[:end // 128]
        assert np.array_equal(form.scales[:want_scales.shape[0], :want_scales.shape[1]].cpu().numpy(), want_scales)
    y = torch.empty(T, C, device="cuda")
    rows = torch.full((d["rows"], C), float("nan"), device="cuda")
    rows[:end] = cuda(v).float()
    ftm.ft_expert_combine(d, s, rows, T, C, y)
    got = y.cpu().numpy()
    for t in range(T):
        here = (want["pair_row"][t] >= 0).sum()
        with np.errstate(invalid="ignore"):
            assert np.allclose(got[t], here * x[t] if here else 0.0, rtol=1e-6, equal_nan=True)


@pytest.mark.parametrize("align", (16, 128))
@pytest.mark.parametrize("order", ("as they come", "mixed", "by magnitude"))
def test_gather_of_every_bf16_value(order, align):
    """bf16 rows go to 8 bits two values at a time: the same forms as of the values in float32, every bit pattern among them
    (signed zeros, subnormals, infinities, quiet and signalling NaNs of both signs), but for the masked tokens'."""
    r, T, C, k = rng(len(order), align), 128, 512, 3
    bits = np.arange(65536, dtype=np.uint16)
    if order == "mixed":
        bits = r.permutation(bits)
    elif order == "by magnitude":
        bits = np.concatenate([bits[:32768], bits[32768:]]).reshape(2, 32768).T.reshape(-1)
    x = cuda(bits.view(np.int16).reshape(T, C)).view(torch.bfloat16)
    wide = torch.from_numpy((bits.astype(np.uint32) << 16).view(np.float32).reshape(T, C)).cuda()
    d, want, s = layout(r, T, 5, k, align)
    end = int(want["off"][-1])
    both = align == 128
    got, ref = ([filled(d["rows"], C)] + [filled(C, d["rows"])] * both for _ in range(2))
    for xs, forms in ((x, got), (wide, ref)):
        ftm.ft_expert_gather(d, s, xs, T, C, row=forms[0], col=forms[1] if both else None)
    token = np.where(want["row_pair"][:end] >= 0, want["row_pair"][:end] // k, 0)
    bad = ~torch.isfinite(wide)[cuda(token)] & cuda(want["row_pair"][:end] >= 0)[:, None]
    for i, (a, b) in enumerate(zip(got, ref)):
        p, q, nan = (a.codes[:end], b.codes[:end], bad) if i == 0 else (a.codes[:, :end], b.codes[:, :end], bad.T)
        assert torch.equal(a.scales, b.scales)
        assert torch.equal(p[~nan], q[~nan])
        assert torch.all((p[nan] & 0x7F) == 0x7F) and torch.all((q[nan] & 0x7F) == 0x7F)


@pytest.mark.parametrize("rt,yt", ((BF16, BF16), (F32, F32), (BF16, F32), (F32, BF16)))
@pytest.mark.parametrize("T,E,k,C", ROWS)
def test_combine_and_gate_gradient(T, E, k, C, rt, yt):
    r = rng(T, E, C, rt, yt, 2)
    d, want, s = layout(r, T, E, k, 16, part=k % 2 == 0 and E > 4)
    rv, rows = matrix(r, d["rows"], C, rt, spread=1)
    rows[int(want["off"][-1]):] = float("nan")      # behind the last group: not read
    bv, base = matrix(r, T, C, yt, spread=1)
    w = r.normal(size=(T, k)).astype(np.float32)
    half = 2.0 ** -8 if yt == BF16 else U
    for weights in (None, w):
        for b in (None, base):
            y = torch.full((T + 1, C), 5.0, dtype=TORCH[yt], device="cuda")
            ftm.ft_expert_combine(d, s, rows, T, C, y, weights=None if weights is None else cuda(weights), base=b)
            v, mag = experts.combine(want, rv, weights, None if b is None else bv)
            assert np.all(np.abs(f64(y[:T]) - v) <= half * np.abs(v) + (1 + half) * (k + 1) * U * mag)
            assert torch.all(y[T] == 5.0)
    again = base.clone()
    ftm.ft_expert_combine(d, s, rows, T, C, again, weights=cuda(w), base=again)
    assert torch.equal(again, y[:T])
    none = want["pair_row"].max(axis=1) < 0          # tokens without rows: zeros, or what was there
    assert torch.equal(again[cuda(none)], base[cuda(none)])

    dv, dy = matrix(r, T, C, yt, spread=1)
    d_w = torch.full((T + 1, k), 5.0, device="cuda")
    ftm.ft_expert_gate_grad(d, s, rows, dy, T, C, d_w)
    v, mag = experts.gate_grad(want, rv, dv)
    assert np.all(np.abs(f64(d_w[:T]) - v) <= max(C, 24) * U * mag) and torch.all(d_w[T] == 5.0)
    assert np.all(f64(d_w[:T])[want["pair_row"] < 0] == 0)


@pytest.mark.parametrize("rt,yt", ((BF16, BF16), (F32, F32), (BF16, F32)))
@pytest.mark.parametrize("T,E,k,C", ((2047, 4, 3, 80), (2048, 4, 3, 80), (2049, 20, 1, 8192), (2050, 20, 7, 1040), (2051, 64, 64, 128),
                                     (2303, 66, 9, 528), (2100, 8, 4, 2064)))
def test_gate_gradient_of_many_tokens(T, E, k, C, rt, yt):
    """One wave a token, and the sizes beside it; pairs of which all, some or none have a row, in lots of every size."""
    r = rng(T, E, C, rt, yt, 23)
    d, want, s = layout(r, T, E, k, 16, part=E >= 20)
    rv, rows = matrix(r, d["rows"], C, rt, spread=1)
    rows[int(want["off"][-1]):] = float("nan")      # behind the last group: not read
    dv, dy = matrix(r, T, C, yt, spread=1)
    none = want["pair_row"].max(axis=1) < 0
    dy[cuda(none)] = float("nan")                   # tokens without rows: zeros whatever they hold
    d_w = torch.full((T + 1, k), 5.0, device="cuda")
    ftm.ft_expert_gate_grad(d, s, rows, dy, T, C, d_w)
    v, mag = experts.gate_grad(want, rv, dv)
    assert np.all(np.abs(f64(d_w[:T]) - v) <= max(C, 24) * U * mag) and torch.all(d_w[T] == 5.0)
    assert np.all(f64(d_w[:T])[want["pair_row"] < 0] == 0)


def test_tables_out_of_range_are_no_pairs_and_no_rows():
    T, E, k, C = 4, 3, 2, 144
    d = desc(E, k, 16, T)
    R = d["rows"]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    x = torch.ones(T, C, device="cuda")
    row_pair = torch.full((R,), 1 << 30, dtype=torch.int32, device="cuda")
    row_pair[:4] = i32([T * k, -5, 3, 0])
    pair_row = i32([[0, R], [-7, 1 << 30], [1, 2], [-(1 << 31), R - 1]])
    s = ftm.SortBuffers.of(row_pair, pair_row, i32([0, 16, 1 << 30, 1 << 30]), i32([4, 1 << 30, 4]), i32([0]))
    out = torch.full((R, C), 7.0, device="cuda")
    row = filled(R, C)
    ftm.ft_expert_gather(d, s, x, T, C, rows=out, row=row)
    assert not out[:2].any() and torch.all(out[2:4] == 1) and not out[4:].any()
    y, d_w = torch.empty(T, C, device="cuda"), torch.empty(T, k, device="cuda")
    rows = torch.arange(R, device="cuda", dtype=torch.float32)[:, None].expand(R, C).contiguous()
    ftm.ft_expert_combine(d, s, rows, T, C, y)
    assert torch.equal(y[:, 0].cpu(), torch.tensor([0.0, 0.0, 3.0, R - 1.0]))
    ftm.ft_expert_gate_grad(d, s, rows, x, T, C, d_w)
    assert torch.equal(d_w.cpu(), C * torch.tensor([[0.0, 0.0], [0, 0], [1, 2], [0, R - 1.0]]))
    # a product over groups that the tables place outside the rows
    wt = {"w": torch.full((E, 32, 256), 0x38, dtype=torch.uint8, device="cuda"), "s": torch.ones(E, 1, 2, device="cuda")}
    form = ftm.ActCodes(R, C)
    form.codes.zero_()
    form.codes[:, :C] = 0x38
    form.scales.fill_(127)
    yr = torch.full((R, 32), 7.0, device="cuda")
    lin = {"out_features": 32, "in_features": C, "x_dtype": ACT, "y_dtype": F32}
    for off, count in (([0, 16, 1 << 30, 1 << 30], [4, 1 << 30, 4]), ([-16, 5, 40, 3], [-1, 9, 9]), ([R, R, R + 64, -1], [9, 9, 9])):
        s = ftm.SortBuffers.of(row_pair, pair_row, i32(off), i32(count), i32([0]))
        ftm.ft_expert_linear(d, lin, wt, form, s, T, yr)
        assert torch.all((yr == 7.0) | (yr == 0.0) | (yr == C))
    torch.cuda.synchronize()


# --------------------------------------------------------------------------------------- products

def expert_weights(r, n, N, K):
    each = [weight(r, N, K) for _ in range(n)]
    return {k: torch.stack([w[k] for w, _ in each]) for k in ("w", "s")}, np.stack([v for _, v in each])


# T, E, k: mean rows of a group from below 1 to 300, and the groups' own from 0 on
GROUPS = ((1, 8, 2), (9, 16, 4), (40, 12, 3), (100, 9, 2), (300, 6, 2), (300, 3, 2), (520, 5, 4))
SHAPES = ((16, 16), (48, 144), (272, 384), (400, 1040), (576, 128))   # N, K


def run_experts(d, s, wt, form, N, K, T, yt):
    y = torch.full((d["rows"], N), 7.0, dtype=TORCH[yt], device="cuda")
    ftm.ft_expert_linear(d, {"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": yt}, wt, form, s, T, y)
    return y


@pytest.mark.parametrize("yt", (BF16, F32))
@pytest.mark.parametrize("align", (16, 128))
@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("T,E,k", GROUPS)
def test_products(T, E, k, N, K, align, yt):
    r = rng(T, E, N, K, align, yt)
    d, want, s = layout(r, T, E, k, align, part=E % 3 == 0)
    wt, w = expert_weights(r, d["local"], N, K)
    xv = matrix(r, d["rows"], K, spread=1)[0]
    form, q = form_of(xv)                      # padding holds values as well: it is not read
    y = run_experts(d, s, wt, form, N, K, T, yt)
    end = int(want["off"][-1])
    v, mag = experts.product(want, q, w)
    assert_product(y[:end], v, mag, K, yt)
    assert not y[:end][cuda(want["row_pair"][:end] < 0)].any()
    assert torch.all(y[end:] == 7.0)
    assert torch.equal(y, run_experts(d, s, wt, form, N, K, T, yt))


@pytest.mark.parametrize("yt", (BF16, F32))
@pytest.mark.parametrize("T,E,k", ((1, 8, 2), (40, 12, 3), (300, 3, 2)))
def test_products_equal_the_dense_ones(T, E, k, yt):
    """A group's rows times its weight are what ft_linear gives, to the arithmetic's accuracy; blocks of scale 0 that meet
    NaN codes add nothing in either."""
    N, K = 144, 528
    r = rng(T, E, yt, 9)
    d, want, s = layout(r, T, E, k, 128)
    wt, w = expert_weights(r, E, N, K)
    wt["s"][:, 0, 2] = 0.0
    w[:, :128, 256:384] = 0.0
    xv = matrix(r, d["rows"], K, spread=1)[0]
    form, q = form_of(xv)
    form.codes[::3, 300] = 0x7F
    q = q.copy()
    q[::3, 300] = 0.0                           # for the rows 0 .. 127 of the weight
    y = run_experts(d, s, wt, form, N, K, T, yt)
    end = int(want["off"][-1])
    v, mag = experts.product(want, q, w)
    assert_product(y[:end, :128], v[:, :128], mag[:, :128], K, yt)
    group = np.searchsorted(want["off"], np.arange(end), side="right") - 1
    met = f64(wt["s"])[group, 1, 2] != 0        # rows 128 .. 143 of the weight have scales of their own
    nan = (want["row_pair"][:end] >= 0) & (np.arange(end) % 3 == 0) & met
    assert np.array_equal(torch.isnan(y[:end, 128:]).all(dim=1).cpu().numpy(), nan) and nan.any()
    assert np.array_equal(torch.isnan(y[:end, 128:]).any(dim=1).cpu().numpy(), nan)
    assert not torch.isnan(y[:end, :128]).any()


@pytest.mark.parametrize("n,N,K", ((1, 16, 16), (3, 48, 144), (5, 272, 128), (2, 400, 1040)))
def test_transposes(n, N, K):
    r = rng(n, N, K, 10)
    wt, w = expert_weights(r, n, N, K)
    kp, np_ = dense.pad128(K), dense.pad128(N)
    t = {"w": torch.full((n, K, np_), 0xA5, dtype=torch.uint8, device="cuda"), "s": torch.full((n, kp // 128, np_ // 128), 9.0, device="cuda")}
    ftm.ft_expert_linear_transpose(n, N, K, wt, t)
    one = {"w": torch.empty(K, np_, dtype=torch.uint8, device="cuda"), "s": torch.empty(kp // 128, np_ // 128, device="cuda")}
    for e in range(n):
        ftm.ft_linear_transpose(N, K, {"w": wt["w"][e], "s": wt["s"][e]}, one)
        assert torch.equal(t["w"][e], one["w"]) and torch.equal(t["s"][e], one["s"])
        v = dense.weight_values(t["w"][e].cpu().numpy(), t["s"][e].cpu().numpy())
        assert np.array_equal(v[:, :N], w[e].T) and not t["w"][e][:, N:].any()


@pytest.mark.parametrize("N,K", ((16, 16), (48, 144), (272, 400), (576, 128)))
@pytest.mark.parametrize("T,E,k", GROUPS)
def test_weight_gradients(T, E, k, N, K):
    r = rng(T, E, N, K, 11)
    d, want, s = layout(r, T, E, k, 128, part=E % 3 == 0)
    n, end = d["local"], int(want["off"][-1])
    real = np.zeros((d["rows"], 1))
    real[:end, 0] = want["row_pair"][:end] >= 0
    dyv, xv = matrix(r, d["rows"], N, spread=1)[0] * real, matrix(r, d["rows"], K, spread=1)[0] * real
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    dc.codes[:, end:], xc.codes[:, end:] = 0x7F, 0x7F           # behind the last group: not read
    v, mag = experts.weight_grad(want, a.T, b.T)
    most = max(1, int(want["count"].max()))
    for dt, kw in ((BF16, {}), (F32, {}), (F32, {"accumulate": True})):
        dw = torch.full((n + 1, N, K), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, dw, **kw)
        assert torch.all(dw[n] == 3.0)
        if kw:
            err = np.abs(f64(dw[:n]) - 3.0 - v)
            assert np.all(err <= (most + most // 128 + 4) * U * (mag + 3.0))
            assert torch.all(dw[:n][cuda(want["count"] == 0)] == 3.0)
        else:
            assert_product(dw[:n], v, mag, most, dt)
            assert not dw[:n][cuda(want["count"] == 0)].any()


def test_weight_gradients_without_tokens():
    d = desc(3, 2, 128, 0)
    for dt in (BF16, F32):
        dw = torch.full((3, 48, 144), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_expert_weight_grad(d, 48, 144, None, None, None, 0, dw)
        assert not dw.any()
    ftm.ft_expert_weight_grad(d, 48, 144, None, None, None, 0, dw.fill_(3.0), accumulate=True)
    assert torch.all(dw == 3.0)


@pytest.mark.parametrize("T,E,k,N,K", ((1922, 3, 2, 4256, 800), (700, 2, 1, 4112, 1808)))
def test_products_and_gradients_of_the_largest_tile(T, E, k, N, K):
    """Groups of many tiles, reductions over 7 and 15 blocks, so that every place of the tile's rings is used again."""
    r = rng(T, N, K, 12)
    d, want, s = layout(r, T, E, k, 128)
    end = int(want["off"][-1])
    wt, w = expert_weights(r, E, N, K)
    real = np.zeros((d["rows"], 1))
    real[:end, 0] = want["row_pair"][:end] >= 0
    xv = matrix(r, d["rows"], K, spread=1)[0] * real
    form, q = form_of(xv)
    v, mag = experts.product(want, q, w)
    assert_product(run_experts(d, s, wt, form, N, K, T, BF16)[:end], v, mag, K, BF16)
    dyv = matrix(r, d["rows"], N, spread=1)[0] * real
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    dw = torch.empty(E, N, K, dtype=torch.bfloat16, device="cuda")
    ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, dw)
    v, mag = experts.weight_grad(want, a.T, b.T)
    assert_product(dw, v, mag, int(want["count"].max()), BF16)


@pytest.mark.parametrize("T,E,k,N,K", ((700, 16, 2, 272, 400), (300, 20, 2, 1040, 272), (60, 200, 2, 272, 272), (20, 1000, 1, 16, 32),
                                       (9000, 16, 2, 48, 144), (40, 34, 1, 2064, 144), (200, 3, 1, 4112, 4112)))
def test_weight_gradients_of_runs_of_experts(T, E, k, N, K):
    """From 16 experts on their columns are read a run of experts ahead: whole and partial runs, runs without any row, bands of
    one to three tiles, tables that leave the runs' order; and many tiles of few experts, which read nothing ahead."""
    r = rng(T, E, N, K, 21)
    skew = routing(r, T, E, k, 4.0)
    d = desc(E, k, 128, T)
    want = experts.sort(skew, 0, E, 128, d["rows"])
    s, end = tables_of(want), int(want["off"][-1])
    real = np.zeros((d["rows"], 1))
    real[:end, 0] = want["row_pair"][:end] >= 0
    dyv, xv = matrix(r, d["rows"], N, spread=1)[0] * real, matrix(r, d["rows"], K, spread=1)[0] * real
    (dc, a), (xc, b) = form_of(dyv.T), form_of(xv.T)
    dc.codes[:, end:], xc.codes[:, end:] = 0x7F, 0x7F
    v, mag = experts.weight_grad(want, a.T, b.T)
    most = max(1, int(want["count"].max()))
    for dt in (BF16, F32):
        dw = torch.full((E + 1, N, K), 3.0, dtype=TORCH[dt], device="cuda")
        ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, dw)
        assert torch.all(dw[E] == 3.0)
        assert_product(dw[:E], v, mag, most, dt)
    if E >= 16:
        s.off.copy_(s.off.flip(0))                              # every group ends before it starts
        ftm.ft_expert_weight_grad(d, N, K, dc, xc, s, T, dw)
        assert not dw[:E].any() and torch.all(dw[E] == 3.0)


@pytest.mark.parametrize("T,E,k,N,K", ((2400, 16, 2, 4352, 272), (2000, 34, 3, 2048, 1040), (1300, 3, 1, 12544, 400)))
def test_products_of_tall_tiles_and_blocks_of_scale_0(T, E, k, N, K):
    """Enough tiles for those of 256 x 128 and 256 x 256; weight blocks of scale 0 meet codes that are NaN."""
    r = rng(T, N, K, 14)
    d, want, s = layout(r, T, E, k, 128)
    end = int(want["off"][-1])
    wt, w = expert_weights(r, E, N, K)
    wt["s"][:, 1::3, 1] = 0.0
    rows = np.arange(N) // 128 % 3 == 1
    w[:, rows, 128:256] = 0.0
    form, q = form_of(matrix(r, d["rows"], K, spread=1)[0])
    v, mag = experts.product(want, q, w)
    assert_product(run_experts(d, s, wt, form, N, K, T, BF16)[:end], v, mag, K, BF16)
    form.codes[::5, 130] = 0x7F
    q = q.copy()
    q[::5, 130] = 0.0
    v, mag = experts.product(want, q, w)
    y = run_experts(d, s, wt, form, N, K, T, BF16)
    dropped = cuda(rows)
    assert_product(y[:end][:, dropped], v[:, rows], mag[:, rows], K, BF16)
    real = cuda((want["row_pair"][:end] >= 0) & (np.arange(end) % 5 == 0))
    assert torch.equal(torch.isnan(y[:end]).any(dim=1), real) and torch.all(y[end:] == 7.0)


@pytest.mark.parametrize("align", (16, 128))
@pytest.mark.parametrize("T,E,k,N,K", ((500, 3, 3, 12416, 144), (560, 3, 3, 12432, 16), (400, 3, 3, 12416, 144), (225, 9, 2, 8176, 144), (90, 9, 5, 8080, 272),
                                       (1500, 3, 1, 16400, 48)))
def test_products_whose_last_round_is_halved(T, E, k, N, K, align):
    """Some tiles more than a multiple of the CUs: tiles of half the features, whose second half may be 16 rows or none."""
    r = rng(T, E, N, K, 22)
    wt, w = expert_weights(r, E, N, K)
    d, want, s = layout(r, T, E, k, align)
    form, q = form_of(matrix(r, d["rows"], K, spread=1)[0])
    end = int(want["off"][-1])
    y = run_experts(d, s, wt, form, N, K, T, BF16)
    v, mag = experts.product(want, q, w)
    assert_product(y[:end], v, mag, K, BF16)
    assert torch.all(y[end:] == 7.0)
    assert not y[:end][cuda(want["row_pair"][:end] < 0)].any()


@pytest.mark.parametrize("T,E,k", ((40, 63, 3), (40, 64, 3), (40, 65, 3), (200, 1000, 4), (3000, 1024, 2)))
def test_many_groups(T, E, k):
    """More groups than lanes: a workgroup finds its tile among them; tables with a bool mask, and with too few rows."""
    N, K = 48, 144
    r = rng(T, E, 15)
    wt, w = expert_weights(r, E, N, K)
    ids, mask = routing(r, T, E, k), r.random(T) < 0.8
    for rows in (None, max(128, ftm.ft_expert_sort_rows({"n_experts": E, "top_k": k, "align": 16}, T) // 3 // 128 * 128)):
        for align in (16, 128):
            d = desc(E, k, align, T, rows=rows)
            s = run_sort(d, ids, mask)
            want = experts.sort(ids, 0, E, align, d["rows"], mask) if T * E < 1e6 else None
            if want is None:
                want = {n: getattr(s, n).cpu().numpy() for n in ("row_pair", "pair_row", "off", "count", "dropped")}
            else:
                assert np.array_equal(s.row_pair.cpu().numpy(), want["row_pair"])
            form, q = form_of(matrix(r, d["rows"], K, spread=1)[0])
            end = int(want["off"][-1])
            v, mag = experts.product(want, q, w)
            for yt in (BF16, F32):
                y = run_experts(d, s, wt, form, N, K, T, yt)
                assert_product(y[:end], v, mag, K, yt)
                assert torch.all(y[end:] == 7.0)
            if align == 128:
                x = torch.where(s.row_pair[:, None] >= 0, cuda(q).float(), torch.zeros(1, device="cuda"))
                xc = ftm.ActCodes(K, d["rows"])
                ftm.ft_act_quantize(x, d["rows"], K, col=xc)
                dw = torch.full((E, K, K), 3.0, device="cuda")
                ftm.ft_expert_weight_grad(d, K, K, xc, xc, s, T, dw)
                vals = dense.values(xc.codes.cpu().numpy(), xc.scales.cpu().numpy())[:, :d["rows"]].T
                v, mag = experts.weight_grad(want, vals, vals)
                assert_product(dw, v, mag, max(1, int(want["count"].max())), F32)


def test_every_token_at_one_expert():
    """The groups are as uneven as they can be: few-row kernels then meet long groups, and the others are empty."""
    T, E, N, K = 130, 64, 272, 400
    d = desc(E, 1, 16, T)
    ids = np.full((T, 1), 37, np.int32)
    s = run_sort(d, ids)
    want = assert_tables(s, d, ids)
    r = rng(13)
    wt, w = expert_weights(r, E, N, K)
    form, q = form_of(matrix(r, d["rows"], K, spread=1)[0])
    for yt in (BF16, F32):
        y = run_experts(d, s, wt, form, N, K, T, yt)
        v, mag = experts.product(want, q, w)
        assert_product(y[:len(v)], v, mag, K, yt)
        assert torch.all(y[len(v):] == 7.0)
