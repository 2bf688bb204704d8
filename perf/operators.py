"""The dense 8-bit product, the 8-bit SwiGLU checkpoint and the router's balance loss: the calls that
are measured, with each operator's plain form.

Every case is one pass through one operator:

``linear``           y = x W^T, x in bf16, W in e4m3fn with one float32 scale per 128 x 128 block; x is
                     quantised per row and 128 channels to e4m3fn with a power-of-two scale
``linear_backward``  from dy in bf16: dx = dy W on the transposed weight, and dW = dy^T x from the 8-bit
                     column form of x that the forward pass kept
``swiglu``           silu(gate) * up in 8 bits, and gate and up kept in 8 bits for the backward pass
``swiglu_backward``  from the kept gate and up and the gradient of h: the gradient of gate and up in the
                     row and the column form, and h in the column form
``balance``          per sequence: routed pairs per expert, mean router probabilities, balance loss
``router_backward``  gradient of the router logits from the balance loss and from the gates

A matrix of R rows and K columns in 8-bit form is codes [R][Kp] (Kp: K up to a multiple of 128, codes
of the padding 0) and e8m0 scale bytes [Kp / 128][Rp]; the column form of a matrix is the form of its
transpose.  The layers are the DeepSeek-V3 (hidden 7168, inter 2048, 256 experts) and Qwen3-30B-A3B
(2048, 768, 128 experts) shapes that the framework is configured for elsewhere.
"""
from __future__ import annotations

import math

import torch

own = False

SOFTMAX, SIGMOID = 0, 1
_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------------------------------- cases

def _linear(T, N, K, y="bf16", **kw):
    return {"op": "linear", "T": T, "N": N, "K": K, "y": y, **kw}


def _linear_backward(T, N, K, dw="bf16", **kw):
    return {"op": "linear_backward", "T": T, "N": N, "K": K, "dw": dw, **kw}


def _swiglu(op, T, I, **kw):
    return {"op": op, "T": T, "I": I, **kw}


def _router(op, T, E, k, gating, n_seq, padded, **kw):
    return {"op": op, "T": T, "E": E, "k": k, "gating": gating, "n_seq": n_seq, "padded": padded, **kw}


def listed():
    return [
        # one user decoding: gate and up projection of the DeepSeek-V3-shaped shared expert
        _linear(1, 4096, 7168, name="linear_decode_1"),
        # an ordinary decode batch through its down projection
        _linear(32, 7168, 2048, name="linear_decode_32"),
        # a ragged prompt chunk through a Qwen3-shaped gate and up projection, kept in float32
        _linear(777, 1536, 2048, y="f32", name="linear_chunk_777"),
        # the largest prompt chunk, and the forward pass of a large training batch
        _linear(8192, 4096, 7168, name="linear_prompt_8192"),
        # a small ragged training batch: both gradients of a Qwen3-shaped projection, the weight's kept
        # in float32 as an optimizer takes it
        _linear_backward(1500, 1536, 2048, dw="f32", name="linear_backward_1500"),
        # a large training batch: both gradients of the DeepSeek-V3-shaped down projection
        _linear_backward(8192, 7168, 2048, name="linear_backward_8192"),
        # a short ragged training batch between the two projections
        _swiglu("swiglu", 300, 2048, name="swiglu_300"),
        # a large training batch on the way back
        _swiglu("swiglu_backward", 8192, 2048, name="swiglu_backward_8192"),
        # the load of one decode batch over the experts
        _router("balance", 48, 128, 8, SOFTMAX, 1, False, name="balance_48"),
        # a packed training batch of several sequences with padding inside
        _router("balance", 8192, 256, 8, SIGMOID, 9, True, name="balance_8192"),
        # a small ragged batch on the way back
        _router("router_backward", 777, 128, 8, SOFTMAX, 1, False, name="router_backward_777"),
        # the largest packed batch on the way back
        _router("router_backward", 65536, 256, 8, SIGMOID, 16, True, name="router_backward_65536"),
    ]


_MAX_FLOPS = 2 * 8192 * 4096 * 7168   # of the largest listed product


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("linear", "linear", "linear_backward", "swiglu", "swiglu_backward", "balance",
                     "router_backward"))
    if op in ("linear", "linear_backward"):
        N, K = 16 * _log(rng, 4, 512), 16 * _log(rng, 8, 512)
        if rng.random() < 0.6:   # most projections are whole blocks
            N, K = max(128, N // 128 * 128), K // 128 * 128
        most = _MAX_FLOPS // (2 * N * K * (2 if op == "linear_backward" else 1))
        T = _log(rng, 1, max(1, min(8192, most)))
        kind = rng.choice(("bf16", "f32"))
        return _linear(T, N, K, y=kind) if op == "linear" else _linear_backward(T, N, K, dw=kind)
    if op in ("swiglu", "swiglu_backward"):
        return _swiglu(op, _log(rng, 1, 8192), 128 * _log(rng, 1, 32))
    E = rng.choice((8, 60, 64, 128, 160, 256, 384, 512))
    T = _log(rng, 1, min(65536, (1 << 24) // E))
    return _router(op, T, E, rng.choice((1, 2, 4, 6, 8)), rng.choice((SOFTMAX, SIGMOID)),
                   min(T, rng.choice((1, 1, 3, 8, 32))), rng.random() < 0.5)


# ---------------------------------------------------------------------------- plain 8-bit forms

def _up128(n):
    return -(-n // 128) * 128


def _quantize(x):
    """(codes [R][Kp], scale bytes [Kp / 128][Rp], both uint8) of x [R][K]: per row and 128 columns the
    smallest power of two that keeps the codes within 448."""
    R, K = x.shape
    b = torch.zeros(R, _up128(K), dtype=torch.float32, device=x.device)
    b[:, :K] = x
    b = b.view(R, -1, 128)
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


def _values(codes, scales, dtype=torch.float32):
    """The values [R][Kp] that an 8-bit form stands for."""
    R = codes.shape[0]
    s = torch.exp2(scales[:, :R].t().to(dtype) - 127)
    return codes.view(torch.float8_e4m3fn).to(torch.float32).to(dtype) * s.repeat_interleave(128, 1)


def _weight_values(w, s, N, K, dtype=torch.float32):
    v = w.view(torch.float8_e4m3fn).to(torch.float32).to(dtype)
    return (v * s.to(dtype).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1))[:, :K]


def _form(codes, scales):
    """An 8-bit form as outputs: the codes' and the scales' values."""
    return {"codes": codes.view(torch.float8_e4m3fn), "scales": scales[:, :codes.shape[0]].view(torch.float8_e8m0fnu)}


# --------------------------------------------------------------------------------------- inputs

def _weight(N, K, g):
    """N(0, 1/sqrt K) in e4m3fn, scale amax / 448 per 128 x 128 block: codes [N][Kp], scales."""
    Np, Kp = _up128(N), _up128(K)
    v = torch.zeros(Np, Kp, device="cuda")
    v[:N, :K] = torch.randn(N, K, generator=g, device="cuda") / math.sqrt(K)
    b = v.view(Np // 128, 128, Kp // 128, 128)
    s = b.abs().amax(dim=(1, 3)) / 448.0
    q = (b / s[:, None, :, None]).clamp_(-448.0, 448.0)
    return q.view(Np, Kp)[:N].to(torch.float8_e4m3fn).view(torch.uint8).contiguous(), s


def _activations(T, C, g):
    """N(0, 1) with a few channels some ten times larger, as hidden states have them."""
    x = torch.randn(T, C, generator=g, device="cuda")
    big = torch.rand(C, generator=g, device="cuda") < 0.01
    return torch.where(big, x * 12.0, x).to(torch.bfloat16)


def _probabilities(logits, gating):
    if gating == SOFTMAX:
        e = torch.exp(logits - logits.amax(dim=1, keepdim=True))
        return e / e.sum(dim=1, keepdim=True)
    s = 1 / (1 + torch.exp(-logits))
    return s / s.sum(dim=1, keepdim=True)


def _sequence_of(st):
    """Sequence index of each token, n_seq for tokens of none (behind the last, or padding)."""
    T, n = st["T"], st["n_seq"]
    seq = torch.bucketize(torch.arange(T, device="cuda"), st["seq_off"].long(), right=True) - 1
    if st["mask"] is not None:
        seq = torch.where(st["mask"] != 0, seq, torch.full_like(seq, n))
    return seq.clamp(max=n)


def _router_inputs(case, g):
    T, E, k, n = case["T"], case["E"], case["k"], case["n_seq"]
    dev = {"device": "cuda"}
    rank = torch.randperm(E, generator=g, **dev).float() + 1
    logits = torch.randn(T, E, generator=g, **dev) - 0.8 * torch.log(rank)
    val, ids = logits.topk(k, dim=1)
    if case["gating"] == SIGMOID:
        val = torch.sigmoid(val)
        gates = val / val.sum(dim=1, keepdim=True)
    else:
        gates = torch.softmax(val, dim=1)
    # ragged sequences; with padding, the last one ends before the batch does and some tokens inside
    # do not count
    cuts = (torch.rand(n - 1, generator=g, **dev) * T).long().sort().values
    end = T - T // 16 if case["padded"] else T
    off = torch.cat((torch.zeros(1, dtype=torch.long, **dev), cuts.clamp(max=end), torch.full((1,), end, **dev)))
    mask = (torch.rand(T, generator=g, **dev) < 0.95).to(torch.uint8) if case["padded"] else None
    st = {**case, "logits": logits, "topk_ids": ids.to(torch.int32), "topk_w": gates, "seq_off": off.to(torch.int32),
          "mask": mask, "coef": 0.01, "d_loss": torch.rand(n, generator=g, **dev) + 0.5,
          "d_topk_w": torch.randn(T, k, generator=g, **dev) * 0.1}
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    op = case["op"]
    st = dict(case)
    if op in ("linear", "linear_backward"):
        T, N, K = case["T"], case["N"], case["K"]
        w, s = _weight(N, K, g)
        if op == "linear":
            st |= {"x": _activations(T, K, g), "w": w, "s": s,
                   "out": torch.empty(T, N, dtype=_DTYPES[case["y"]], device="cuda")}
        else:
            # the transposed weight and the forward pass's column form of x, as a training loop keeps them
            wt = torch.zeros(K, _up128(N), dtype=torch.uint8, device="cuda")
            wt[:, :N] = w.t()[:K]
            st |= {"wt": wt, "st": s.t().contiguous(), "x_col": _quantize(_activations(T, K, g).float().t()),
                   "dy": (_activations(T, N, g).float() * 1e-3).to(torch.bfloat16),
                   "dx": torch.empty(T, K, dtype=torch.bfloat16, device="cuda"),
                   "dw_out": torch.empty(N, K, dtype=_DTYPES[case["dw"]], device="cuda")}
    elif op in ("swiglu", "swiglu_backward"):
        gu = _activations(case["T"], 2 * case["I"], g)
        if op == "swiglu":
            st["gu"] = gu
        else:
            st |= {"saved": _quantize(gu.float()), "dh": (_activations(case["T"], case["I"], g).float() * 1e-3).to(torch.bfloat16)}
    else:
        st = _router_inputs(case, g)
        if op == "router_backward":
            st |= _plain_balance(st)
            st["d_logits"] = torch.zeros_like(st["logits"])
    return st


# ---------------------------------------------------------------------------------- plain forms

def _plain_linear(st):
    x = _values(*_quantize(st["x"].float()))[:, :st["K"]]
    return (x @ _weight_values(st["w"], st["s"], st["N"], st["K"]).t()).to(st["out"].dtype)


def _plain_linear_backward(st):
    dy = st["dy"].float()
    T, N, K = st["T"], st["N"], st["K"]
    dx = _values(*_quantize(dy))[:, :N] @ _weight_values(st["wt"], st["st"], K, N).t()
    dw = _values(*_quantize(dy.t()))[:, :T] @ _values(*st["x_col"])[:, :T].t()
    return {"dx": dx.to(torch.bfloat16), "dw": dw.to(_DTYPES[st["dw"]])}


def _plain_swiglu(st):
    gu = st["gu"].float()
    gate, up = gu[:, :st["I"]], gu[:, st["I"]:]
    h = gate / (1 + torch.exp(-gate)) * up
    return {"h": _form(*_quantize(h)), "saved": _form(*_quantize(gu))}


def _plain_swiglu_backward(st):
    gu, dh = _values(*st["saved"]), st["dh"].float()
    gate, up = gu[:, :st["I"]], gu[:, st["I"]:]
    sig = 1 / (1 + torch.exp(-gate))
    dgu = torch.cat((dh * up * sig * (1 + gate * (1 - sig)), dh * gate * sig), dim=1)
    return {"dgu_row": _form(*_quantize(dgu)), "dgu_col": _form(*_quantize(dgu.t())),
            "h_col": _form(*_quantize((gate * sig * up).t()))}


def _plain_balance(st):
    T, E, k, n = st["T"], st["E"], st["k"], st["n_seq"]
    # member [n + 1][T]: which tokens a sequence counts; sums over up to T tokens in 64 bits
    member = (torch.arange(n + 1, device="cuda")[:, None] == _sequence_of(st)[None, :]).double()
    tokens = member.sum(dim=1)
    prob = member @ _probabilities(st["logits"], st["gating"]).double()
    selected = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    selected = selected.scatter_add_(1, st["topk_ids"].long(), torch.ones(T, k, dtype=torch.float64, device="cuda"))
    counts = member @ selected
    some = tokens[:n].clamp(min=1)[:, None]
    prob, counts = prob[:n] / some, counts[:n]
    frac = st["coef"] * E * counts / (k * some)
    return {"counts": counts.to(torch.int32), "tokens": tokens[:n].to(torch.int32), "prob": prob.float(),
            "frac": frac.float(), "loss": (frac * prob).sum(dim=1).float()}


def _plain_router_backward(st):
    seq = _sequence_of(st)
    n = st["n_seq"]
    logits, ids, gates, dg = st["logits"], st["topk_ids"].long(), st["topk_w"], st["d_topk_w"]
    counted = (seq < n)[:, None]
    s = seq.clamp(max=n - 1)
    p = _probabilities(logits, st["gating"])
    a = torch.ones_like(logits) if st["gating"] == SOFTMAX else 1 / (1 + torch.exp(logits))
    frac = st["frac"][s]
    weight = (st["d_loss"] / st["tokens"].clamp(min=1))[s][:, None]
    d = torch.where(counted, weight * p * a * (frac - (frac * p).sum(dim=1, keepdim=True)), torch.zeros_like(p))
    dgate = gates * a.gather(1, ids) * (dg - (gates * dg).sum(dim=1, keepdim=True))
    d = d.scatter_add(1, ids, dgate)
    # rows behind the last sequence stay as they were
    return torch.where((torch.arange(st["T"], device="cuda") < st["seq_off"][-1])[:, None], d, st["d_logits"])


# ---------------------------------------------------------------------------- the framework's calls

def _own(st):
    import paper_2608_16157_amd as ftm

    op, T = st["op"], st["T"]
    if op == "linear":
        desc = {"out_features": st["N"], "in_features": st["K"], "x_dtype": ftm.FT_DT_BF16,
                "y_dtype": ftm.FT_DT_BF16 if st["y"] == "bf16" else ftm.FT_DT_F32}
        if "ws" not in st:
            st["ws"] = ftm.alloc_linear_workspace(desc, T)
        ftm.ft_linear(desc, {"w": st["w"], "s": st["s"]}, st["x"], T, st["out"], st["ws"])
        return st["out"]
    if op == "linear_backward":
        N, K = st["N"], st["K"]
        if "row" not in st:
            st["row"], st["col"] = ftm.ActCodes(T, N), ftm.ActCodes(N, T)
        ftm.ft_act_quantize(st["dy"], T, N, st["row"], st["col"])
        ftm.ft_linear({"out_features": K, "in_features": N, "x_dtype": ftm.FT_DT_FP8_ACT, "y_dtype": ftm.FT_DT_BF16},
                      {"w": st["wt"], "s": st["st"]}, st["row"], T, st["dx"])
        ftm.ft_linear_weight_grad(N, K, T, st["col"], _own_form(st["x_col"], K, T), st["dw_out"])
        return {"dx": st["dx"], "dw": st["dw_out"]}
    if op == "swiglu":
        if "h" not in st:
            st["h"], st["saved"] = ftm.ActCodes(T, st["I"]), ftm.ActCodes(T, 2 * st["I"])
        ftm.ft_swiglu_quantize(st["gu"], T, st["I"], st["h"], st["saved"])
        return {n: _form(st[n].codes, st[n].scales) for n in ("h", "saved")}
    if op == "swiglu_backward":
        I = st["I"]
        if "dgu_row" not in st:
            st |= {"dgu_row": ftm.ActCodes(T, 2 * I), "dgu_col": ftm.ActCodes(2 * I, T), "h_col": ftm.ActCodes(I, T)}
        ftm.ft_swiglu_backward(_own_form(st["saved"], T, 2 * I), st["dh"], T, I, st["dgu_row"], st["dgu_col"], st["h_col"])
        return {n: _form(st[n].codes, st[n].scales) for n in ("dgu_row", "dgu_col", "h_col")}
    desc = {"n_experts": st["E"], "top_k": st["k"], "gating": st["gating"], "n_seq": st["n_seq"], "coef": st["coef"]}
    if op == "balance":
        if "bal" not in st:
            st["bal"], st["ws"] = ftm.BalanceBuffers(st["n_seq"], st["E"]), ftm.alloc_balance_workspace(desc, T)
        ftm.ft_balance_loss(desc, st["logits"], st["topk_ids"], T, st["bal"], st["ws"], seq_off=st["seq_off"], mask=st["mask"])
        return {n: getattr(st["bal"], n) for n in ("counts", "tokens", "prob", "frac", "loss")}
    if "bal" not in st:
        st["bal"] = ftm.BalanceBuffers.of(st["counts"], st["tokens"], st["prob"], st["frac"], st["loss"])
    ftm.ft_router_backward(desc, st["logits"], st["topk_ids"], T, st["bal"], st["d_loss"], st["d_logits"],
                           topk_w=st["topk_w"], d_topk_w=st["d_topk_w"], seq_off=st["seq_off"], mask=st["mask"])
    return st["d_logits"]


def _own_form(form, rows, cols):
    import paper_2608_16157_amd as ftm

    return ftm.ActCodes.of(form[0], form[1], rows, cols)


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "linear_backward": _plain_linear_backward, "swiglu": _plain_swiglu,
            "swiglu_backward": _plain_swiglu_backward, "balance": _plain_balance,
            "router_backward": _plain_router_backward}[state["op"]](state)


# ------------------------------------------------------------------------------ work, definition

def work(case):
    op, T = case["op"], case["T"]
    if op in ("linear", "linear_backward"):
        N, K = case["N"], case["K"]
        wb = N * K + 4 * (_up128(N) // 128) * (_up128(K) // 128)
        if op == "linear":
            return {"bytes": 2 * T * K + wb + T * N * (2 if case["y"] == "bf16" else 4), "flops": 2 * T * N * K}
        return {"bytes": 2 * T * N + wb + 2 * T * K + T * K + T * K // 128 + N * K * (2 if case["dw"] == "bf16" else 4), "flops": 4 * T * N * K}
    if op == "swiglu":
        return {"bytes": T * case["I"] * 7 + 3 * T * case["I"] // 128, "flops": 6 * T * case["I"]}
    if op == "swiglu_backward":
        return {"bytes": T * case["I"] * 9 + 7 * T * case["I"] // 128, "flops": 14 * T * case["I"]}
    E, k = case["E"], case["k"]
    if op == "balance":
        return {"bytes": 4 * T * E + 4 * T * k + 12 * case["n_seq"] * E, "flops": 5 * T * E}
    return {"bytes": 8 * T * E + 12 * T * k + 4 * case["n_seq"] * E, "flops": 9 * T * E}


def _exact_quantize(x):
    """The 8-bit form of x in 64 bits, from its definition: 2^e with the smallest e such that 448 * 2^e
    covers the block, values to the nearest e4m3fn value, ties to even."""
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


def exact(case, seed):
    st = prepare(case, seed)
    op, T = case["op"], case["T"]

    def value(q):
        return q["codes"] * q["scales"].t().repeat_interleave(128, 1)

    def weight(w, s):
        R, C = w.shape
        blocks = torch.arange(R, device="cuda") // 128, torch.arange(C, device="cuda") // 128
        return w.view(torch.float8_e4m3fn).double() * s.double()[blocks[0]][:, blocks[1]]

    if op == "linear":
        return value(_exact_quantize(st["x"].double())) @ weight(st["w"], st["s"]).t()
    if op == "linear_backward":
        dy = st["dy"].double()
        x_col = st["x_col"][0].view(torch.float8_e4m3fn).double() * torch.exp2(
            st["x_col"][1][:, :case["K"]].double() - 127).t().repeat_interleave(128, 1)
        return {"dx": value(_exact_quantize(dy)) @ weight(st["wt"], st["st"]).t(),
                "dw": value(_exact_quantize(dy.t())) @ x_col.t()}
    if op == "swiglu":
        gate, up = st["gu"].double().chunk(2, dim=1)
        return {"h": _exact_quantize(torch.nn.functional.silu(gate) * up), "saved": _exact_quantize(st["gu"].double())}
    if op == "swiglu_backward":
        gu = (st["saved"][0].view(torch.float8_e4m3fn).double() * torch.exp2(
            st["saved"][1][:, :T].double() - 127).t().repeat_interleave(128, 1)).requires_grad_(True)
        gate, up = gu.chunk(2, dim=1)
        h = torch.nn.functional.silu(gate) * up
        (dgu,) = torch.autograd.grad(h, gu, st["dh"].double())
        return {"dgu_row": _exact_quantize(dgu), "dgu_col": _exact_quantize(dgu.t()), "h_col": _exact_quantize(h.detach().t())}

    # the router in 64 bits, sequence by sequence; its gradient from the definition by differentiation
    E, k, n = case["E"], case["k"], case["n_seq"]
    back = op == "router_backward"
    logits = st["logits"].double().requires_grad_(back)
    p = torch.softmax(logits, 1) if case["gating"] == SOFTMAX else torch.sigmoid(logits)
    if case["gating"] == SIGMOID:
        p = p / p.sum(1, keepdim=True)
    off = st["seq_off"].tolist()
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if st["mask"] is None else st["mask"] != 0
    counts, tokens, probs, fracs, losses = [], [], [], [], []
    for s in range(n):
        rows = torch.arange(off[s], off[s + 1], device="cuda")
        rows = rows[keep[rows]]
        m = max(1, rows.numel())
        c = torch.bincount(st["topk_ids"][rows].flatten().long(), minlength=E)
        counts.append(c)
        tokens.append(rows.numel())
        probs.append(p[rows].sum(0) / m)
        fracs.append(st["coef"] * E * c.double() / (k * m))
        losses.append((fracs[-1] * probs[-1]).sum())
    if not back:
        return {"counts": torch.stack(counts).to(torch.int32), "tokens": torch.tensor(tokens, dtype=torch.int32),
                "prob": torch.stack(probs), "frac": torch.stack(fracs), "loss": torch.stack(losses)}
    sel = logits.gather(1, st["topk_ids"].long())
    gates = torch.softmax(sel, 1) if case["gating"] == SOFTMAX else torch.sigmoid(sel)
    if case["gating"] == SIGMOID:
        gates = gates / gates.sum(1, keepdim=True)
    live = torch.arange(T, device="cuda") < off[-1]
    total = (torch.stack(losses) * st["d_loss"].double()).sum() + (gates * st["d_topk_w"].double())[live].sum()
    (d,) = torch.autograd.grad(total, logits)
    return d
