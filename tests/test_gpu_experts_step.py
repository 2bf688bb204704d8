"""A training step of a layer's routed experts through the library's calls as a program makes them: norm, router, sort,
gather, products, SwiGLU, combine, norm with gates, and all of it back, the router's logits included.

Against the same layer in 64 bits without 8-bit forms, differentiated by torch on the CPU.  Tolerance: rounding to e4m3fn is
off by at most 2^-4 of a value, evenly spread over its step, so 2^-4 / sqrt(3) / 1.44 = 0.025 of a matrix's norm; on the
longest way (x, kept gate and up, h, dy, d_gate and d_up) five of them add up as unrelated errors and SwiGLU's
second derivative at most doubles them: 0.025 sqrt(5) 2 = 0.11 of a gradient's norm, 0.16 allowed.  The gradients of the
gates are inner products over a token's channels, which may cancel: an error of 0.16 of one vector's norm changes the
product by up to 0.16 of the two norms' product (Cauchy and Schwarz), and that is what theirs are held to.  A softmax's
d_logit_j = g_j (dg_j - sum g_i dg_i) is off by at most twice the largest error of a dg (g_j <= 1, sum g = 1; a
sigmoid's further factor is at most 1).  Captured and replayed steps equal eager ones bit for bit."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_16157_amd as ftm
import workloads
from tests.test_gpu_dense import ACT, BF16, F32, cuda, f64

pytestmark = pytest.mark.gpu


class Step:
    """Buffers and calls of one step over T tokens; the experts first .. first + local - 1 are here."""

    def __init__(self, T, E, k, H, I, gating, seed, masked=False, align=128, first=0, local=None):
        lay = workloads.random_layer(seed, hidden=H, inter=I, n_experts=E, top_k=k, tokens=T, gating=gating,
                                     w_dtype=workloads.DT_FP8, n_resident=E, zipf_s=0.7)
        self.T, self.E, self.k, self.H, self.I, self.gating, self.lay = T, E, k, H, I, gating, lay
        r = np.random.default_rng(seed)
        slot = lay.slot_table.long()
        local = E if local is None else local
        here = slice(first, first + local)
        pick = lambda t: t.view(torch.uint8)[slot][here].cuda().contiguous() if t.dtype != torch.float32 else t[slot][here].cuda().contiguous()
        self.w13 = {"w": pick(lay.w13), "s": pick(lay.s13)}
        self.w2 = {"w": pick(lay.w2), "s": pick(lay.s2)}
        new = lambda *s, dtype=torch.bfloat16: torch.empty(*s, dtype=dtype, device="cuda")
        self.wt13 = {"w": new(local, H, 2 * I, dtype=torch.uint8), "s": new(local, H // 128, 2 * I // 128, dtype=torch.float32)}
        self.wt2 = {"w": new(local, I, H, dtype=torch.uint8), "s": new(local, I // 128, H // 128, dtype=torch.float32)}
        ftm.ft_expert_linear_transpose(local, 2 * I, H, self.w13, self.wt13)
        ftm.ft_expert_linear_transpose(local, H, I, self.w2, self.wt2)
        self.logits = lay.logits.cuda()
        self.x = cuda(r.normal(size=(T, H))).to(torch.bfloat16)
        self.dr = cuda(r.normal(size=(T, H))).to(torch.bfloat16)
        self.mask = cuda((r.random(T) < 0.8).astype(np.uint8)) if masked else None
        self.params = {"pre": cuda(r.normal(size=H) * 0.1 + 1).float(), "post": cuda(r.normal(size=H) * 0.1 + 1).float(),
                       "gate": cuda(r.normal(size=H) * 0.3 + 1).float(), "token_gate": cuda(r.random(T) + 0.5).float()}
        kinds = {"channels": H, "x_dtype": BF16, "y_dtype": BF16, "w_dtype": F32, "eps": 1e-5}
        self.before, self.after = kinds, {**kinds, "post_norm": 1, "scale": 0.5}
        self.d = {"n_experts": E, "top_k": k, "first": first, "local": local, "align": align}
        self.d["rows"] = rows = ftm.ft_expert_sort_rows(self.d, T)
        self.route, self.ws_route = ftm.RouteBuffers(T, k, E), ftm.alloc_workspace(self.route_desc(), T)
        self.sort, self.ws_sort = ftm.SortBuffers(self.d, T), ftm.alloc_sort_workspace(self.d, T)
        self.ws_norm = ftm.alloc_block_norm_workspace(self.after, T)
        self.slots = torch.arange(E, dtype=torch.int32, device="cuda")
        self.n, self.b, self.r = new(T, H), new(T, H), new(T, H)
        form = lambda R, K: ftm.ActCodes(R, K)
        self.xr, self.xc, self.h, self.saved = form(rows, H), form(H, rows), form(rows, I), form(rows, 2 * I)
        self.gu, self.y = new(rows, 2 * I), new(rows, H)
        self.db, self.dn, self.dx = new(T, H), new(T, H), new(T, H)
        self.dyr, self.dyc = form(rows, H), form(H, rows)
        self.dh, self.dxr = new(rows, I), new(rows, H)
        self.dgr, self.dgc, self.hc = form(rows, 2 * I), form(2 * I, rows), form(I, rows)
        self.dw13, self.dw2 = new(local, 2 * I, H, dtype=torch.float32), new(local, H, I, dtype=torch.float32)
        self.d_topk_w, self.d_logits = new(T, k, dtype=torch.float32), new(T, E, dtype=torch.float32)
        f32 = lambda n: new(n, dtype=torch.float32)
        self.grads_after = {"post": f32(H), "gate": f32(H), "token_gate": f32(T)}
        self.grads_before = {"pre": f32(H)}
        for t in (self.gu, self.y, self.dh, self.dxr):      # rows that no call writes may hold anything
            t.fill_(float("nan"))
        for c in (self.xr, self.xc, self.h, self.saved, self.dyr, self.dyc, self.dgr, self.dgc, self.hc):
            c.codes.fill_(0x7F)
            c.scales.fill_(0xFF)

    def route_desc(self):
        return {"hidden": self.H, "inter": self.I, "n_experts": self.E, "top_k": self.k, "gating": self.gating, "w_dtype": ftm.FT_DT_FP8E4M3FN_B128,
                "x_dtype": BF16, "n_slots": self.E, "shared_slot": -1, "combine": 0, "act_quant": 0}

    def linear(self, N, K):
        return {"out_features": N, "in_features": K, "x_dtype": ACT, "y_dtype": BF16}

    def forward(self, training=True):
        T, H, I, d, s = self.T, self.H, self.I, self.d, self.sort
        ftm.ft_block_norm(self.before, self.params, self.x, None, T, n=self.n)
        ftm.ft_route_only(self.route_desc(), self.logits, self.slots, T, self.route, self.ws_route)
        ids, self.gates = self.route.topk_ids.view(-1)[:T * self.k], self.route.topk_w.view(-1)[:T * self.k]
        ftm.ft_expert_sort(d, ids, T, s, self.ws_sort, mask=self.mask)
        ftm.ft_expert_gather(d, s, self.n, T, H, row=self.xr, col=self.xc if training else None)
        ftm.ft_expert_linear(d, self.linear(2 * I, H), self.w13, self.xr, s, T, self.gu)
        ftm.ft_swiglu_quantize(self.gu, d["rows"], I, self.h, self.saved if training else None)
        ftm.ft_expert_linear(d, self.linear(H, I), self.w2, self.h, s, T, self.y)
        ftm.ft_expert_combine(d, s, self.y, T, H, self.b, weights=self.gates)
        ftm.ft_block_norm(self.after, self.params, self.x, self.b, T, r=self.r)

    def backward(self):
        T, H, I, d, s = self.T, self.H, self.I, self.d, self.sort
        ftm.ft_block_norm_backward(self.after, self.params, self.r, self.b, self.dr, None, T, self.dx, self.db, self.grads_after, self.ws_norm)
        ftm.ft_expert_gather(d, s, self.db, T, H, weights=self.gates, row=self.dyr, col=self.dyc)
        ftm.ft_expert_gate_grad(d, s, self.y, self.db, T, H, self.d_topk_w)
        bal = {"n_experts": self.E, "top_k": self.k, "gating": self.gating, "n_seq": 1}
        ftm.ft_router_backward(bal, self.logits, self.route.topk_ids, T, None, None, self.d_logits, topk_w=self.gates, d_topk_w=self.d_topk_w)
        ftm.ft_expert_linear(d, self.linear(I, H), self.wt2, self.dyr, s, T, self.dh)
        ftm.ft_swiglu_backward(self.saved, self.dh, d["rows"], I, self.dgr, self.dgc, self.hc)
        ftm.ft_expert_weight_grad(d, H, I, self.dyc, self.hc, s, T, self.dw2)
        ftm.ft_expert_linear(d, self.linear(H, 2 * I), self.wt13, self.dgr, s, T, self.dxr)
        ftm.ft_expert_weight_grad(d, 2 * I, H, self.dgc, self.xc, s, T, self.dw13)
        ftm.ft_expert_combine(d, s, self.dxr, T, H, self.dn)
        # in front of the block there was no block: the residual's gradient goes through, plus the norm's
        ftm.ft_block_norm_backward(self.before, self.params, self.x, None, self.dx, self.dn, T, self.dx, None, self.grads_before, self.ws_norm)

    def outputs(self):
        return {"r": self.r, "b": self.b, "dx": self.dx, "dw13": self.dw13, "dw2": self.dw2, "d_logits": self.d_logits,
                "pre": self.grads_before["pre"], **self.grads_after}

    def run(self):
        self.forward()
        self.backward()


def reference(st):
    """The outputs in 64 bits, differentiated by torch; for inner products ("inner") the norms' products per token."""
    E, k, H, I = st.E, st.k, st.H, st.I
    first, local = st.d["first"], st.d["local"]

    def values(w, n, N, K):
        codes = w["w"].cpu().view(torch.float8_e4m3fn).double()[:, :N, :K]
        s = w["s"].cpu().double().repeat_interleave(128, 1)[:, :N].repeat_interleave(128, 2)[:, :, :K]
        return (codes * s).requires_grad_(True)

    leaf = lambda t: t.detach().cpu().double().requires_grad_(True)
    w13, w2 = values(st.w13, local, 2 * I, H), values(st.w2, local, H, I)
    x, logits = leaf(st.x), leaf(st.logits)
    p = {n: leaf(t) for n, t in st.params.items()}
    ids = st.route.topk_ids.view(-1)[:st.T * k].view(st.T, k).cpu().long()
    sel = logits.gather(1, ids)
    gates = torch.softmax(sel, 1) if st.gating == oracle.GATE_SOFTMAX else torch.sigmoid(sel) / torch.sigmoid(sel).sum(1, keepdim=True)
    unit = lambda v: v / torch.sqrt((v * v).mean(1, keepdim=True) + 1e-5)
    n = p["pre"] * unit(x)
    b = torch.zeros(st.T, H, dtype=torch.float64)
    live = torch.ones(st.T) if st.mask is None else st.mask.cpu()
    largest = torch.zeros(st.T, dtype=torch.float64)      # norm of a token's rows of the experts
    for t in range(st.T):
        for j in range(k):
            e = int(ids[t, j]) - first
            if live[t] and 0 <= e < local:
                gate, up = (w13[e] @ n[t]).split(I)
                y = w2[e] @ (torch.nn.functional.silu(gate) * up)
                largest[t] = max(largest[t], y.detach().norm())
                b[t] = b[t] + gates[t, j] * y
    u = p["post"] * unit(b)
    r = x + 0.5 * p["gate"] * p["token_gate"][:, None] * u
    leaves = {"dx": x, "dw13": w13, "dw2": w2, "d_logits": logits, **p, "db": b}
    dr = st.dr.cpu().double()
    grads = dict(zip(leaves, torch.autograd.grad((r * dr).sum(), list(leaves.values()))))
    inner = {"token_gate": (0.5 * p["gate"] * dr).norm(dim=1) * u.norm(dim=1), "d_logits": 2 * grads["db"].norm(dim=1) * largest}
    return {"r": r.detach(), "b": b.detach(), **grads, "inner": {n: v.detach().numpy() for n, v in inner.items()}}


CASES = ((40, 8, 2, 256, 128, 0, False), (130, 12, 3, 384, 256, 1, True), (300, 6, 2, 256, 384, 0, True), (1, 4, 2, 128, 128, 1, False))


@pytest.mark.parametrize("T,E,k,H,I,gating,masked", CASES)
def test_step_against_autograd(T, E, k, H, I, gating, masked):
    st = Step(T, E, k, H, I, gating, 5, masked)
    st.run()
    want = reference(st)
    for n, t in st.outputs().items():
        got, ref = f64(t), want[n].numpy()
        if n in want["inner"]:
            off = np.abs(got - ref).reshape(T, -1).max(axis=1)
            assert np.all(off <= 0.16 * want["inner"][n] + 1e-12), (n, float((off / want["inner"][n]).max()))
        else:
            err = np.linalg.norm(got - ref) / max(np.linalg.norm(ref), 1e-30)
            assert err <= 0.16, (n, err)
    first = {n: t.clone() for n, t in st.outputs().items()}
    st.run()
    assert all(torch.equal(first[n], t) for n, t in st.outputs().items())


def test_parts_of_the_experts_add_up():
    """Every expert on one of three GPUs: the sum of the partial outputs and gradients is the whole."""
    T, E, k, H, I = 90, 9, 3, 256, 128
    whole = Step(T, E, k, H, I, 0, 8)
    whole.run()
    b, dn, d_gates = (torch.zeros_like(t, dtype=torch.float64) for t in (whole.b, whole.dn, whole.d_topk_w))
    for first in (0, 3, 6):
        part = Step(T, E, k, H, I, 0, 8, first=first, local=3)
        part.forward()
        b += part.b.double()
        # the block's output is known only once it is added up; then the same gradient reaches every part
        part.r, part.b = whole.r, whole.b
        part.backward()
        dn += part.dn.double()
        d_gates += part.d_topk_w.double()
        assert torch.equal(part.dw13, whole.dw13[first:first + 3]) and torch.equal(part.dw2, whole.dw2[first:first + 3])
    # up to three roundings to bf16 in place of one
    assert np.all(np.abs(f64(whole.b) - f64(b)) <= 2.0 ** -8 * 4 * np.abs(f64(whole.b)).max())
    assert np.all(np.abs(f64(whole.dn) - f64(dn)) <= 2.0 ** -8 * 4 * np.abs(f64(whole.dn)).max())
    assert torch.equal(whole.d_topk_w.double(), d_gates)


@pytest.mark.parametrize("T", (5, 70, 300))
def test_forward_against_the_layer_call(T):
    """ft_moe_forward with 8-bit activations over the same weights: its h is rounded to bf16 in front of the 8 bits where
    here gate and up are, so an h may round to the next code: 2^-3 of it, for the share of them that lies 2^-8 from a
    border (2^-3): 2^-3 sqrt(2^-3) = 0.044 of the norm at the most."""
    E, k, H, I = 8, 2, 256, 256
    st = Step(T, E, k, H, I, 0, 9, align=16)
    st.forward(training=False)
    desc = {**st.route_desc(), "act_quant": ftm.FT_ACT_FP8_1x128_POW2}
    banks = {"w13": st.w13["w"], "w2": st.w2["w"], "s13": st.w13["s"], "s2": st.w2["s"]}
    out, route = torch.empty(T, H, device="cuda"), ftm.RouteBuffers(T, k, E)
    ftm.ft_moe_forward(desc, banks, st.logits, st.slots, st.n, T, out, route, ftm.alloc_workspace(desc, T))
    assert torch.equal(route.topk_ids, st.route.topk_ids)
    assert np.linalg.norm(f64(st.b) - f64(out)) <= 0.044 * np.linalg.norm(f64(out))


def test_captured_step_replays_with_other_routings():
    """The whole step in one graph, replayed with other inputs, eager work and synchronisations in between, and a second
    graph over the same workspaces: every replay equals the eager step on the same inputs."""
    st = Step(130, 12, 3, 256, 128, 0, 11, True)
    st.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    for part in (st.run, lambda: (st.forward(), st.backward())):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            part()
        graphs.append(g)
    torch.cuda.current_stream().wait_stream(side)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for i in range(4):
        st.logits.copy_(torch.randn(st.logits.shape, generator=gen, device="cuda"))
        st.x.copy_(torch.randn(st.x.shape, generator=gen, device="cuda"))
        if i == 2:
            st.mask.zero_()                      # nothing is routed
        if i == 3:
            st.mask.fill_(1)
            st.logits[:, 3] += 50.0              # everything at one expert, among others
        st.run()
        want = {n: t.clone() for n, t in st.outputs().items()}
        torch.cuda.synchronize()
        for g in graphs:
            for t in st.outputs().values():
                t.fill_(9.0)
            g.replay()
            assert all(torch.equal(want[n], t) for n, t in st.outputs().items())
        if i == 2:
            assert not st.dw13.any() and not st.dw2.any() and not st.b.any()


def test_two_steps_on_two_streams_at_once():
    a, b = Step(200, 8, 2, 256, 128, 0, 21), Step(170, 8, 2, 256, 128, 1, 22)
    want = []
    for st in (a, b):
        st.run()
        want.append({n: t.clone() for n, t in st.outputs().items()})
        for t in st.outputs().values():
            t.fill_(9.0)
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        for st, s in zip((a, b), streams):
            with torch.cuda.stream(s):
                st.run()
    torch.cuda.synchronize()
    for st, w in zip((a, b), want):
        assert all(torch.equal(w[n], t) for n, t in st.outputs().items())
