"""The routed experts in training and the norms around them: the calls that are measured, with each operator's
plain form.

Every case is one pass through one operator:

``dispatch``          the routed (token, expert) pairs sorted by expert, and the tokens' rows gathered in
                      that order: as they are, or in 8 bits in the row form (the next product's input) and
                      in the column form (kept for the weight's gradient)
``combine``           the experts' rows back to their tokens, times their gates, on top of what is there
``combine_backward``  from the gradient of the combined rows: the gradient of the experts' rows in both
                      8-bit forms, and the gradient of the gates
``experts``           y = x W_e^T for every row x of expert e's group; x in 8 bits, W in e4m3fn with one
                      float32 scale per 128 x 128 block
``experts_backward``  from dy in both 8-bit forms: dx = dy W_e on the transposed weights, and
                      dW_e = dy^T x over the rows of each group
``norm``              after a block: r = x + scale g_c h_t (p_c b / rms(b)), and before the next one:
                      n = w_c r / rms(r), in bf16 and in the row form; rms(v) = sqrt(mean v^2 + eps)
``norm_backward``     from the gradients of r and n: those of x, b, the two weights and the two gates

Groups of rows start at multiples of ``align``; the rows that fill one up are zeros, rows behind the last
group stay as they were.  8-bit forms: blocks of 128 in e4m3fn with a power-of-two scale, codes [R][Kp]
(Kp: K up to a multiple of 128) and e8m0 scale bytes [Kp / 128][Rp]; the column form of a matrix is the
form of its transpose.  The layers are the DeepSeek-V3 (hidden 7168, inter 2048, 256 experts, 32 of them
where they are spread over eight GPUs) and Qwen3-30B-A3B (2048, 768, 128 experts) shapes that the framework
is configured for elsewhere.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_EPS = 1e-6


# ---------------------------------------------------------------------------------------- cases

def _rows_case(op, T, E, k, local, C, **kw):
    """``local`` of the E experts are here; C channels; ``masked``: some tokens are padding."""
    return {"op": op, "T": T, "E": E, "k": k, "local": local, "C": C, "masked": False, **kw}


def _experts(op, T, E, k, local, N, K, out, **kw):
    return {"op": op, "T": T, "E": E, "k": k, "local": local, "N": N, "K": K, "out": out, "masked": False, **kw}


def _norm(op, T, C, x, post, **kw):
    return {"op": op, "T": T, "C": C, "x": x, "post": post, **kw}


def listed():
    return [
        # a few users decoding: their rows for the product over the experts
        _rows_case("dispatch", 4, 256, 8, 256, 7168, forms="row", name="dispatch_decode_4"),
        # a large training batch, padding inside: rows of the forward pass and what the backward pass keeps
        _rows_case("dispatch", 8192, 256, 8, 256, 7168, forms="both", masked=True, name="dispatch_train_8192"),
        # a decode batch back to its tokens, on top of the shared expert's output
        _rows_case("combine", 32, 256, 8, 256, 7168, y="bf16", base=True, name="combine_decode_32"),
        # a large training batch back to its tokens
        _rows_case("combine", 8192, 256, 8, 256, 7168, y="bf16", base=False, name="combine_train_8192"),
        # a small ragged training batch on the way back
        _rows_case("combine_backward", 1500, 128, 8, 128, 2048, name="combine_backward_1500"),
        # a decode batch through the gate and up projections of its experts
        _experts("experts", 16, 128, 8, 128, 1536, 2048, "bf16", name="experts_decode_16"),
        # a large batch through gate and up on one of eight GPUs that share the experts
        _experts("experts", 32768, 256, 8, 32, 4096, 7168, "bf16", name="experts_train_32768"),
        # both gradients of a small ragged training batch, the weight's in float32 as an optimizer takes it
        _experts("experts_backward", 1500, 128, 8, 128, 1536, 2048, "f32", name="experts_backward_1500"),
        # both gradients of the down projection for a large batch on one of eight GPUs
        _experts("experts_backward", 16384, 256, 8, 32, 7168, 2048, "bf16", name="experts_backward_16384"),
        # one decoding step between two blocks
        _norm("norm", 4, 7168, "bf16", False, name="norm_decode_4"),
        # a ragged prompt chunk, the residual stream in float32, a norm on both sides of the block
        _norm("norm", 777, 2048, "f32", True, name="norm_chunk_777"),
        # a large training batch on the way back
        _norm("norm_backward", 8192, 7168, "bf16", True, name="norm_backward_8192"),
    ]


# of the largest listed cases
_MAX_ELEMENTS = 8192 * 8 * 7168
_MAX_WEIGHT = 32 * 4096 * 7168
_MAX_FLOPS = 2 * 32768 * 4096 * 7168
_MAX_NORM = 8192 * 7168


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(("dispatch", "combine", "combine_backward", "experts", "experts_backward", "norm", "norm_backward"))
    if op in ("norm", "norm_backward"):
        C = 16 * _log(rng, 4, 1024)
        return _norm(op, _log(rng, 1, min(32768, _MAX_NORM // C)), C, rng.choice(("bf16", "f32")), rng.random() < 0.5)
    E = rng.choice((8, 60, 64, 128, 160, 256, 384, 512))
    k = rng.choice((1, 2, 4, 6, 8))
    local = max(1, E // rng.choice((1, 1, 4, 8)))
    masked = rng.random() < 0.3
    if op in ("experts", "experts_backward"):
        local = min(local, 128)
        N, K = 16 * _log(rng, 8, 256), 16 * _log(rng, 8, 448)
        if rng.random() < 0.6:   # most projections are whole blocks
            N, K = max(128, N // 128 * 128), max(128, K // 128 * 128)
        while local > 1 and local * N * K > _MAX_WEIGHT // 2:
            local //= 2
        each = 2 * N * K * k * local / E * (2 if op == "experts_backward" else 1)
        T = _log(rng, 1, min(32768, _MAX_FLOPS // 2 / each, 65536 * E / (k * local)))
        return _experts(op, T, E, k, local, N, K, rng.choice(("bf16", "f32")), masked=masked)
    C = 16 * _log(rng, 8, 512)
    T = _log(rng, 1, min(65536, _MAX_ELEMENTS // 2 / (k * C)))
    case = _rows_case(op, T, E, k, local, C, masked=masked)
    if op == "dispatch":
        case["forms"] = rng.choice(("plain", "row", "both"))
    elif op == "combine":
        case |= {"y": rng.choice(("bf16", "f32")), "base": rng.random() < 0.5}
    return case


def _align(case):
    """Column forms take whole blocks of 128 rows per group; without them 16 keep the padding small."""
    return 128 if case["op"] in ("combine_backward", "experts_backward") or case.get("forms") == "both" or \
        case["T"] * case["k"] >= 64 * case["E"] else 16


def _capacity(case):
    """Rows for every pair whatever the routing; where the experts are spread over GPUs, for twice the
    even share."""
    a, pairs, local = _align(case), case["T"] * case["k"], case["local"]
    if local < case["E"]:
        pairs = min(pairs, 2 * pairs * local // case["E"] + 64)
    return max(a, (pairs + min(local, pairs) * (a - 1)) // a * a)


# ---------------------------------------------------------------------------- plain 8-bit forms

def _up128(n):
    return -(-n // 128) * 128


def _quantize(x):
    """(codes [R][Kp], scale bytes [Kp / 128][Rp], both uint8) of x [R][K]: per row and 128 columns the
    smallest power of two that keeps the codes within 448."""
    R, K = x.shape
    b = torch.nn.functional.pad(x, (0, _up128(K) - K)).view(R, -1, 128)
    amax = b.abs().amax(dim=2)
    m, e = torch.frexp(amax)
    e = torch.where(amax > 0, e - 9 + (m > 0.875).to(e.dtype), torch.zeros_like(e)).clamp(-127, 127)
    # the factor in two halves: 2^-127 alone is no normal float32
    half = torch.div(-e, 2, rounding_mode="floor")
    v = torch.ldexp(torch.ldexp(b, half[:, :, None]), (-e - half)[:, :, None])
    codes = v.to(torch.float8_e4m3fn).view(torch.uint8).view(R, -1)
    scales = torch.full((b.shape[1], _up128(R)), 127, dtype=torch.uint8, device=x.device)
    scales[:, :R] = (e + 127).to(torch.uint8).t()
    return codes, scales


def _values(codes, scales):
    """The values [R][Kp] that an 8-bit form stands for."""
    s = torch.exp2(scales[:, :codes.shape[0]].t().float() - 127)
    return codes.view(torch.float8_e4m3fn).float() * s.repeat_interleave(128, 1)


def _weight_values(w, s, N, K):
    """[n][N][K] of n experts' codes [n][N][Kp] and scales."""
    v = w.view(torch.float8_e4m3fn).float()
    return (v * s.repeat_interleave(128, 1)[:, :N].repeat_interleave(128, 2))[:, :, :K]


def _form(codes, scales):
    """An 8-bit form as outputs: the codes' and the scales' values."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales[:, :codes.shape[0]].view(torch.float8_e8m0fnu)}


# --------------------------------------------------------------------------------------- inputs

def _weights(n, N, K, g):
    """N(0, 1/sqrt K) in e4m3fn, scale amax / 448 per 128 x 128 block, for n experts."""
    Np, Kp = _up128(N), _up128(K)
    v = torch.zeros(n, Np, Kp, device="cuda")
    v[:, :N, :K] = torch.randn(n, N, K, generator=g, device="cuda") / math.sqrt(K)
    b = v.view(n, Np // 128, 128, Kp // 128, 128)
    s = b.abs().amax(dim=(2, 4)) / 448.0
    q = (b / s[:, :, None, :, None]).clamp_(-448.0, 448.0)
    return q.view(n, Np, Kp)[:, :N].to(torch.float8_e4m3fn).view(torch.uint8).contiguous(), s


def _activations(T, C, g):
    """N(0, 1) with a few channels some ten times larger, as hidden states have them."""
    x = torch.randn(T, C, generator=g, device="cuda")
    big = torch.rand(C, generator=g, device="cuda") < 0.01
    return torch.where(big, x * 12.0, x).to(torch.bfloat16)


def _routing(case, g):
    """Experts of unequal popularity, their gates, and which tokens count."""
    T, E, k = case["T"], case["E"], case["k"]
    rank = torch.randperm(E, generator=g, device="cuda").float() + 1
    val, ids = (torch.randn(T, E, generator=g, device="cuda") - 0.5 * torch.log(rank)).topk(k, dim=1)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.95).to(torch.uint8) if case["masked"] else None
    return {"topk_ids": ids.to(torch.int32), "topk_w": torch.softmax(val, dim=1), "mask": mask}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op, T = case["op"], case["T"]
    if op in ("norm", "norm_backward"):
        return _prepare_norm(case, g)
    first = case["E"] // case["local"] // 2 * case["local"]
    st = {**case, **_routing(case, g), "align": _align(case), "rows": _capacity(case), "first": first}
    rows = st["rows"]
    if op == "dispatch":
        C = case["C"]
        st["x"] = _activations(T, C, g)
        # what the call writes into; it leaves rows behind the last group alone
        if case["forms"] == "plain":
            st["out"] = torch.zeros(rows, C, dtype=torch.bfloat16, device="cuda")
        else:
            for name, R, K in (("row", rows, C), ("col", C, rows))[:2 if case["forms"] == "both" else 1]:
                st[name] = (torch.zeros(R, _up128(K), dtype=torch.uint8, device="cuda"),
                            torch.zeros(_up128(K) // 128, _up128(R), dtype=torch.uint8, device="cuda"))
        return st
    st |= _plain_sort(st)
    used = (torch.arange(rows, device="cuda") < st["off"][-1])[:, None]
    real = (st["row_pair"] >= 0)[:, None]
    if op == "combine":
        st["expert_rows"] = _activations(rows, case["C"], g) * used
        st["y_out"] = torch.empty(T, case["C"], dtype=_DTYPES[case["y"]], device="cuda")
        st["base_in"] = _activations(T, case["C"], g).to(_DTYPES[case["y"]]) if case["base"] else None
    elif op == "combine_backward":
        C = case["C"]
        st["expert_rows"] = _activations(rows, C, g) * used
        st["dy"] = (_activations(T, C, g).float() * 1e-3).to(torch.bfloat16)
        for name, R, K in (("row", rows, C), ("col", C, rows)):
            st[name] = (torch.zeros(R, _up128(K), dtype=torch.uint8, device="cuda"),
                        torch.zeros(_up128(K) // 128, _up128(R), dtype=torch.uint8, device="cuda"))
    else:
        N, K, n = case["N"], case["K"], case["local"]
        w, s = _weights(n, N, K, g)
        # a training program's host has the groups' sizes of the step, as every one does that calls a product per expert
        st["starts"], st["filled"] = st["off"].tolist(), st["count"].tolist()
        if op == "experts":
            st |= {"w": w, "s": s, "x_row": _quantize((_activations(rows, K, g) * real).float()),
                   "y_out": torch.zeros(rows, N, dtype=_DTYPES[case["out"]], device="cuda")}
        else:
            # the transposed weights and the forward pass's column form of x, as a training loop keeps them
            wt = torch.zeros(n, K, _up128(N), dtype=torch.uint8, device="cuda")
            wt[:, :, :N] = w.transpose(1, 2)[:, :K]
            dy = _activations(rows, N, g).float() * 1e-3 * real
            st |= {"wt": wt, "st": s.transpose(1, 2).contiguous(), "dy_row": _quantize(dy), "dy_col": _quantize(dy.t()),
                   "x_col": _quantize((_activations(rows, K, g) * real).float().t()),
                   "dx": torch.zeros(rows, K, dtype=torch.bfloat16, device="cuda"),
                   "dw": torch.empty(n, N, K, dtype=_DTYPES[case["out"]], device="cuda")}
    return st


def _prepare_norm(case, g):
    T, C, kind = case["T"], case["C"], _DTYPES[case["x"]]
    dev = {"device": "cuda"}
    st = {**case, "scale": 0.5, "block": _activations(T, C, g),
          "pre": 1 + 0.1 * torch.randn(C, generator=g, **dev), "gate": 0.3 * torch.randn(C, generator=g, **dev),
          "token_gate": torch.rand(T, generator=g, **dev),
          "post": 1 + 0.1 * torch.randn(C, generator=g, **dev) if case["post"] else None}
    x = torch.randn(T, C, generator=g, **dev) * 3
    x = (x + 20 * (torch.rand(C, generator=g, **dev) < 0.005)).to(kind)
    if case["op"] == "norm":
        return {**st, "x_in": x, "r": torch.empty_like(x), "n": torch.empty(T, C, dtype=torch.bfloat16, **dev),
                "row": (torch.zeros(T, _up128(C), dtype=torch.uint8, **dev),
                        torch.zeros(_up128(C) // 128, _up128(T), dtype=torch.uint8, **dev))}
    return {**st, "r": x, "dr": (torch.randn(T, C, generator=g, **dev) * 1e-3).to(kind),
            "dn": (_activations(T, C, g).float() * 1e-3).to(torch.bfloat16),
            "dx": torch.empty_like(x), "db": torch.empty(T, C, dtype=torch.bfloat16, **dev),
            "d_token_gate": torch.empty(T, **dev), "d_pre": torch.empty(C, **dev), "d_gate": torch.empty(C, **dev),
            "d_post": torch.empty(C, **dev) if case["post"] else None}


# ---------------------------------------------------------------------------------- plain forms

def _plain_sort(st):
    T, k, n, a, rows = st["T"], st["k"], st["local"], st["align"], st["rows"]
    dev = {"device": "cuda"}
    key = st["topk_ids"].long() - st["first"]
    here = (key >= 0) & (key < n)
    if st["mask"] is not None:
        here = here & (st["mask"] != 0)[:, None]
    key = torch.where(here, key, torch.full_like(key, n)).view(-1)
    pairs = torch.zeros(n + 1, dtype=torch.long, **dev).scatter_add_(0, key, torch.ones_like(key))
    before = torch.cumsum(pairs, 0) - pairs
    off = torch.cumsum(torch.cat((pairs.new_zeros(1), (pairs[:n] + a - 1) // a * a)), 0).clamp(max=rows)
    count = torch.minimum(pairs[:n], rows - off[:n])
    key, order = torch.sort(key, stable=True)
    rank = torch.arange(T * k, **dev) - before[key]
    e = key.clamp(max=n - 1)
    kept = (key < n) & (rank < count[e])
    row = torch.where(kept, off[e] + rank, torch.full_like(rank, rows))
    row_pair = torch.full((rows + 1,), -1, dtype=torch.long, **dev).scatter_(0, row, order)
    pair_row = torch.empty_like(row).scatter_(0, order, torch.where(kept, row, torch.full_like(row, -1)))
    return {"row_pair": row_pair[:rows].to(torch.int32), "pair_row": pair_row.view(T, k).to(torch.int32),
            "off": off.to(torch.int32), "count": count.to(torch.int32),
            "dropped": (pairs[:n].sum() - count.sum()).to(torch.int32).view(1)}


def _gathered(x, row_pair, k, weights=None):
    """float32 rows in the groups' order, zeros where a row has no pair."""
    p = row_pair.long().clamp(min=0)
    v = x.float()[p // k]
    if weights is not None:
        v = v * weights.view(-1)[p][:, None]
    return torch.where((row_pair >= 0)[:, None], v, torch.zeros_like(v))


def _into(out, codes, scales, used_rows, used_blocks):
    """The rows (row form) or the blocks (column form) of the groups, the others as they were in ``out``."""
    if used_rows is not None:
        R = codes.shape[0]
        scales = scales[:, :R].where(used_rows[None, :], out[1][:, :R])
        return _form(codes.where(used_rows[:, None], out[0]), scales)
    return _form(codes.where(used_blocks.repeat_interleave(128)[None, :], out[0]),
                 scales.where(used_blocks[:, None], out[1]))


def _plain_forms(v, off, row, col):
    used = torch.arange(v.shape[0], device="cuda") < off[-1]
    forms = {"row": _into(row, *_quantize(v), used, None)}
    if col is not None:
        forms["col"] = _into(col, *_quantize(v.t()), None, used[::128])
    return forms


def _plain_dispatch(st):
    s = _plain_sort(st)
    v = _gathered(st["x"], s["row_pair"], st["k"])
    if st["forms"] == "plain":
        used = (torch.arange(st["rows"], device="cuda") < s["off"][-1])[:, None]
        return {**s, "rows": v.to(torch.bfloat16).where(used, st["out"])}
    return {**s, **_plain_forms(v, s["off"], st["row"], st.get("col"))}


def _of_pairs(st, rows):
    """[T][k][C] float32 rows of the pairs, zeros for those without."""
    at = st["pair_row"].long()
    v = rows.float()[at.clamp(min=0)]
    return torch.where((at >= 0)[:, :, None], v, torch.zeros_like(v))


def _plain_combine(st):
    y = (_of_pairs(st, st["expert_rows"]) * st["topk_w"][:, :, None]).sum(dim=1)
    if st["base_in"] is not None:
        y = y + st["base_in"].float()
    return y.to(_DTYPES[st["y"]])


def _plain_combine_backward(st):
    v = _gathered(st["dy"], st["row_pair"], st["k"], st["topk_w"])
    d = (_of_pairs(st, st["expert_rows"]) * st["dy"].float()[:, None, :]).sum(dim=2)
    return {**_plain_forms(v, st["off"], st["row"], st["col"]), "d_topk_w": d}


def _behind(out, v):
    """v's rows, and behind them those that ``out`` has."""
    return torch.cat((v.to(out.dtype), out[v.shape[0]:]))


def _plain_experts(st):
    w = _weight_values(st["w"], st["s"], st["N"], st["K"])
    x, o = _values(*st["x_row"])[:, :st["K"]], st["starts"]
    return _behind(st["y_out"], torch.cat([x[o[e]:o[e + 1]] @ w[e].t() for e in range(st["local"])]))


def _plain_experts_backward(st):
    N, K, o = st["N"], st["K"], st["starts"]
    wt = _weight_values(st["wt"], st["st"], K, N)
    dy = _values(*st["dy_row"])[:, :N]
    dx = torch.cat([dy[o[e]:o[e + 1]] @ wt[e].t() for e in range(st["local"])])
    dyc, xc = _values(*st["dy_col"]), _values(*st["x_col"])
    dw = torch.stack([dyc[:, o[e]:o[e + 1]] @ xc[:, o[e]:o[e + 1]].t() for e in range(st["local"])])
    return {"dx": _behind(st["dx"], dx), "dw": dw.to(_DTYPES[st["out"]])}


def _rms(v):
    return torch.sqrt((v * v).mean(dim=1, keepdim=True) + _EPS)


def _plain_norm(st):
    b = st["block"].float()
    if st["post"] is not None:
        b = st["post"] * (b / _rms(b))
    r = st["x_in"].float() + st["scale"] * st["gate"] * st["token_gate"][:, None] * b
    n = st["pre"] * (r / _rms(r))
    return {"r": r.to(st["x_in"].dtype), "n": n.to(torch.bfloat16), "row": _form(*_quantize(n))}


def _plain_norm_backward(st):
    r, b, dn = st["r"].float(), st["block"].float(), st["dn"].float()
    gate, h = st["gate"], st["token_gate"][:, None]
    rr = _rms(r)
    rh, g = r / rr, dn * st["pre"]
    d = st["dr"].float() + (g - rh * (g * rh).mean(dim=1, keepdim=True)) / rr
    q = st["scale"] * gate * h * d
    out = {"dx": d.to(st["r"].dtype), "d_pre": (dn * rh).double().sum(dim=0).float()}
    u, db = b, q
    if st["post"] is not None:
        rb = _rms(b)
        bh, v = b / rb, q * st["post"]
        u, db = st["post"] * bh, (v - bh * (v * bh).mean(dim=1, keepdim=True)) / rb
        out["d_post"] = (q * bh).double().sum(dim=0).float()
    out["db"] = db.to(torch.bfloat16)
    out["d_gate"] = (st["scale"] * h * d * u).double().sum(dim=0).float()
    out["d_token_gate"] = (st["scale"] * gate * d * u).sum(dim=1)
    return out


# ---------------------------------------------------------------------------- the framework's calls

def _desc(st):
    return {"n_experts": st["E"], "top_k": st["k"], "first": st["first"], "local": st["local"], "align": st["align"],
            "rows": st["rows"]}


def _own_form(form, rows, cols):
    import paper_2608_16157_amd as ftm

    return ftm.ActCodes.of(form[0], form[1], rows, cols)


def _own_sort(st):
    import paper_2608_16157_amd as ftm

    if "sort" not in st:
        st["sort"] = ftm.SortBuffers.of(st["row_pair"], st["pair_row"], st["off"], st["count"], st["dropped"])
    return st["sort"]


def _own(st):
    import paper_2608_16157_amd as ftm

    op, T = st["op"], st["T"]
    if op in ("norm", "norm_backward"):
        return _own_norm(st)
    desc, rows = _desc(st), st["rows"]
    if op == "dispatch":
        C = st["C"]
        if "sort" not in st:
            st["sort"], st["ws"] = ftm.SortBuffers(desc, T), ftm.alloc_sort_workspace(desc, T)
            st["forms_out"] = {n: _own_form(st[n], R, K) for n, R, K in (("row", rows, C), ("col", C, rows)) if n in st}
        s = st["sort"]
        ftm.ft_expert_sort(desc, st["topk_ids"], T, s, st["ws"], mask=st["mask"])
        ftm.ft_expert_gather(desc, s, st["x"], T, C, rows=st.get("out"), **st["forms_out"])
        out = {n: getattr(s, n) for n in ("row_pair", "pair_row", "off", "count", "dropped")}
        if "out" in st:
            return {**out, "rows": st["out"]}
        return {**out, **{n: _form(*st[n]) for n in st["forms_out"]}}
    s = _own_sort(st)
    if op == "combine":
        ftm.ft_expert_combine(desc, s, st["expert_rows"], T, st["C"], st["y_out"], weights=st["topk_w"], base=st["base_in"])
        return st["y_out"]
    if op == "combine_backward":
        C = st["C"]
        if "d_topk_w" not in st:
            st["d_topk_w"] = torch.empty_like(st["topk_w"])
        ftm.ft_expert_gather(desc, s, st["dy"], T, C, weights=st["topk_w"], row=_own_form(st["row"], rows, C),
                             col=_own_form(st["col"], C, rows))
        ftm.ft_expert_gate_grad(desc, s, st["expert_rows"], st["dy"], T, C, st["d_topk_w"])
        return {"row": _form(*st["row"]), "col": _form(*st["col"]), "d_topk_w": st["d_topk_w"]}
    N, K = st["N"], st["K"]
    linear = {"x_dtype": ftm.FT_DT_FP8_ACT}
    if op == "experts":
        linear |= {"out_features": N, "in_features": K, "y_dtype": ftm.FT_DT_BF16 if st["out"] == "bf16" else ftm.FT_DT_F32}
        ftm.ft_expert_linear(desc, linear, {"w": st["w"], "s": st["s"]}, _own_form(st["x_row"], rows, K), s, T, st["y_out"])
        return st["y_out"]
    linear |= {"out_features": K, "in_features": N, "y_dtype": ftm.FT_DT_BF16}
    ftm.ft_expert_linear(desc, linear, {"w": st["wt"], "s": st["st"]}, _own_form(st["dy_row"], rows, N), s, T, st["dx"])
    ftm.ft_expert_weight_grad(desc, N, K, _own_form(st["dy_col"], N, rows), _own_form(st["x_col"], K, rows), s, T, st["dw"])
    return {"dx": st["dx"], "dw": st["dw"]}


def _own_norm(st):
    import paper_2608_16157_amd as ftm

    T, C = st["T"], st["C"]
    desc = {"channels": C, "x_dtype": ftm.FT_DT_BF16 if st["x"] == "bf16" else ftm.FT_DT_F32, "y_dtype": ftm.FT_DT_BF16,
            "w_dtype": ftm.FT_DT_F32, "post_norm": st["post"] is not None, "eps": _EPS, "scale": st["scale"]}
    params = {n: st[n] for n in ("pre", "post", "gate", "token_gate")}
    if st["op"] == "norm":
        ftm.ft_block_norm(desc, params, st["x_in"], st["block"], T, st["r"], st["n"], _own_form(st["row"], T, C))
        return {"r": st["r"], "n": st["n"], "row": _form(*st["row"])}
    if "ws" not in st:
        st["ws"] = ftm.alloc_block_norm_workspace(desc, T)
    grads = {"pre": st["d_pre"], "post": st["d_post"], "gate": st["d_gate"], "token_gate": st["d_token_gate"]}
    ftm.ft_block_norm_backward(desc, params, st["r"], st["block"], st["dr"], st["dn"], T, st["dx"], st["db"], grads, st["ws"])
    out = {"dx": st["dx"], "d_pre": st["d_pre"]}
    if st["post"] is not None:
        out["d_post"] = st["d_post"]
    return {**out, "db": st["db"], "d_gate": st["d_gate"], "d_token_gate": st["d_token_gate"]}


def run(state):
    if own:
        return _own(state)
    return {"dispatch": _plain_dispatch, "combine": _plain_combine, "combine_backward": _plain_combine_backward,
            "experts": _plain_experts, "experts_backward": _plain_experts_backward, "norm": _plain_norm,
            "norm_backward": _plain_norm_backward}[state["op"]](state)


# ------------------------------------------------------------------------------ work, definition

def work(case):
    op, T = case["op"], case["T"]
    if op in ("norm", "norm_backward"):
        n, x = T * case["C"], 2 if case["x"] == "bf16" else 4
        if op == "norm":
            return {"bytes": n * (2 * x + 5) + n // 128, "flops": 12 * n}
        return {"bytes": n * (3 * x + 6), "flops": 30 * n}
    pairs = T * case["k"]
    rows = pairs * case["local"] // case["E"]   # an even share of the pairs is here
    if op in ("experts", "experts_backward"):
        N, K, n = case["N"], case["K"], case["local"]
        hit = min(n, rows)   # experts whose weights are read at the least
        wb = hit * (N * K + N * K // 4096)
        if op == "experts":
            return {"bytes": wb + rows * K + rows * N * (2 if case["out"] == "bf16" else 4), "flops": 2 * rows * N * K}
        return {"bytes": wb + rows * (2 * N + K + 2 * K) + n * N * K * (2 if case["out"] == "bf16" else 4), "flops": 4 * rows * N * K}
    C = case["C"]
    if op == "dispatch":
        size = {"plain": 2, "row": 1, "both": 2}[case["forms"]]
        return {"bytes": min(T, rows) * C * 2 + rows * C * size + 12 * pairs, "flops": 4 * rows * C}
    if op == "combine":
        y = 2 if case["y"] == "bf16" else 4
        return {"bytes": rows * C * 2 + T * C * y * (2 if case["base"] else 1) + 8 * pairs, "flops": 2 * rows * C}
    return {"bytes": min(T, rows) * C * 2 + rows * C * 4 + 12 * pairs, "flops": 6 * rows * C}


def _exact_quantize(x):
    """The values of the 8-bit form of x in 64 bits, from its definition: 2^e with the smallest e such that
    448 * 2^e covers the block, values to the nearest e4m3fn value, ties to even."""
    R, K = x.shape
    b = torch.nn.functional.pad(x, (0, _up128(K) - K)).view(R, -1, 128)
    amax = b.abs().amax(dim=2)
    e = torch.ceil(torch.log2(amax.clamp(min=2.0 ** -200) / 448.0))
    e = torch.where(amax <= 448.0 * torch.exp2(e - 1), e - 1, torch.where(amax > 448.0 * torch.exp2(e), e + 1, e))
    e = torch.where(amax > 0, e, torch.zeros_like(e)).clamp(-127, 127)
    v = b / torch.exp2(e)[:, :, None]
    # spacing of the values: 2^(floor(log2 |v|) - 3), at least 2^-9
    step = torch.exp2((torch.frexp(v).exponent.double() - 1).clamp(min=-6.0) - 3)
    return {"codes": (torch.round(v / step) * step).view(R, -1), "scales": torch.exp2(e).t()}


def _exact_sort(case, st):
    """The groups, expert by expert on the host."""
    T, k, n, a, rows = case["T"], case["k"], case["local"], st["align"], st["rows"]
    ids = st["topk_ids"].cpu().numpy().reshape(-1).astype(np.int64) - st["first"]
    if st["mask"] is not None:
        ids = np.where(np.repeat(st["mask"].cpu().numpy() != 0, k), ids, -1)
    row_pair, pair_row = np.full(rows, -1, np.int32), np.full(T * k, -1, np.int32)
    off, count, dropped = np.zeros(n + 1, np.int32), np.zeros(n, np.int32), 0
    for e in range(n):
        pairs = np.nonzero(ids == e)[0]
        at = int(off[e])
        got = pairs[:rows - at]
        row_pair[at:at + len(got)] = got
        pair_row[got] = at + np.arange(len(got))
        count[e], dropped = len(got), dropped + len(pairs) - len(got)
        off[e + 1] = min(rows, at + -(-len(pairs) // a) * a)
    to = lambda v: torch.from_numpy(v).cuda()
    return {"row_pair": to(row_pair), "pair_row": to(pair_row.reshape(T, k)), "off": to(off), "count": to(count),
            "dropped": torch.tensor([dropped], dtype=torch.int32, device="cuda")}


def _exact_rows(x, s, k, weights=None):
    """[rows][C] in 64 bits, built from the pairs' side."""
    at = s["pair_row"].view(-1).long()
    p = torch.nonzero(at >= 0).view(-1)
    v = x.double()[p // k]
    if weights is not None:
        v = v * weights.double().view(-1)[p][:, None]
    out = torch.zeros(s["row_pair"].shape[0], x.shape[1], dtype=torch.float64, device="cuda")
    out[at[p]] = v
    return out


def _exact_forms(v, end, col):
    """8-bit forms of the groups' rows; behind them the forms hold zero bytes (a scale byte of 0 is 2^-127)."""
    row = _exact_quantize(v)
    row["scales"][:, end:] = 2.0 ** -127
    forms = {"row": row}
    if col:
        forms["col"] = _exact_quantize(v.t())
        full = torch.ones(forms["col"]["scales"].shape[0], _up128(v.shape[1]), dtype=torch.float64, device="cuda")
        full[:, :v.shape[1]] = forms["col"]["scales"]
        full[end // 128:] = 2.0 ** -127
        forms["col"]["scales"] = full[:, :v.shape[1]]
    return forms


def exact(case, seed):
    st = prepare(case, seed)
    op, T = case["op"], case["T"]
    if op in ("norm", "norm_backward"):
        return _exact_norm(case, st)
    k = case["k"]
    s = _exact_sort(case, st)
    end = int(s["off"][-1])
    if op == "dispatch":
        v = _exact_rows(st["x"], s, k)
        return {**s, **({"rows": v} if case["forms"] == "plain" else _exact_forms(v, end, case["forms"] == "both"))}
    if op in ("combine", "combine_backward"):
        # pair by pair of a token, in 64 bits
        at, rows = s["pair_row"].long(), st["expert_rows"].double()
        zero = torch.zeros(1, dtype=torch.float64, device="cuda")
        pair = lambda j: torch.where((at[:, j] >= 0)[:, None], rows[at[:, j].clamp(min=0)], zero)
        if op == "combine":
            y = st["base_in"].double() if case["base"] else torch.zeros(T, case["C"], dtype=torch.float64, device="cuda")
            for j in range(k):
                y = y + st["topk_w"][:, j:j + 1].double() * pair(j)
            return y
        dy = st["dy"].double()
        return {**_exact_forms(_exact_rows(st["dy"], s, k, st["topk_w"]), end, True),
                "d_topk_w": torch.stack([(pair(j) * dy).sum(1) for j in range(k)], dim=1)}

    def form(q):
        return q[0].view(torch.float8_e4m3fn).double() * torch.exp2(q[1][:, :q[0].shape[0]].double() - 127).t().repeat_interleave(128, 1)

    def weight(w, scale):
        R, C = w.shape
        blocks = torch.arange(R, device="cuda") // 128, torch.arange(C, device="cuda") // 128
        return w.view(torch.float8_e4m3fn).double() * scale.double()[blocks[0]][:, blocks[1]]

    def product(x, w, scales, N):
        y = torch.zeros(st["rows"], N, dtype=torch.float64, device="cuda")
        for e in range(case["local"]):
            a = int(s["off"][e])
            b = a + int(s["count"][e])
            y[a:b] = x[a:b] @ weight(w[e], scales[e]).t()
        return y

    N, K = case["N"], case["K"]
    if op == "experts":
        return product(form(st["x_row"]), st["w"], st["s"], N)
    dx = product(form(st["dy_row"]), st["wt"], st["st"], K)
    dy, x = form(st["dy_col"]), form(st["x_col"])
    dw = torch.zeros(case["local"], N, K, dtype=torch.float64, device="cuda")
    for e in range(case["local"]):
        a = int(s["off"][e])
        b = a + int(s["count"][e])
        dw[e] = dy[:, a:b] @ x[:, a:b].t()
    return {"dx": dx, "dw": dw}


def _exact_norm(case, st):
    """Forward from the definition; backward by differentiating it."""
    back = case["op"] == "norm_backward"
    leaf = lambda t: None if t is None else t.double().requires_grad_(back)
    b, pre, post, gate, h = (leaf(st[n]) for n in ("block", "pre", "post", "gate", "token_gate"))
    u = b if post is None else torch.nn.functional.normalize(b, dim=1, eps=0) * post * math.sqrt(case["C"])
    if post is not None:   # with eps in the root
        ms = (b * b).mean(1, keepdim=True)
        u = u * torch.sqrt(ms / (ms + _EPS))
    step = st["scale"] * torch.outer(h, gate) * u
    if back:
        # x is what makes r the given one
        x = (st["r"].double() - step).detach().requires_grad_(True)
        r = x + step
    else:
        r = st["x_in"].double() + step
    n = r * pre / ((r * r).mean(1, keepdim=True) + _EPS) ** 0.5
    if not back:
        return {"r": r, "n": n, "row": _exact_quantize(n)}
    total = (r * st["dr"].double()).sum() + (n * st["dn"].double()).sum()
    leaves = [x, pre, b, gate, h] + ([post] if post is not None else [])
    d = torch.autograd.grad(total, leaves)
    out = {"dx": d[0], "d_pre": d[1]}
    if post is not None:
        out["d_post"] = d[5]
    return {**out, "db": d[2], "d_gate": d[3], "d_token_gate": d[4]}
