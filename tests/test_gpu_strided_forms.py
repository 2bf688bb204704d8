"""Weight gradients from column forms whose tensors are strided views, as a program has them that quantised a transposed
matrix or keeps its forms inside a larger buffer: bit for bit those of the same forms in rows."""
import pytest
import torch

import paper_2608_16157_amd as ftm
from tests.test_gpu_dense import form_of, matrix, rng
from tests.test_gpu_experts import layout

pytestmark = pytest.mark.gpu


def transposed(c):
    """The same values as the transposes of buffers in rows."""
    turn = lambda t: t.t().contiguous().t()
    return ftm.ActCodes.of(turn(c.codes), turn(c.scales), c.rows, c.cols)


def sliced(c):
    """The same values inside wider buffers, which hold other bytes around them."""
    def inside(t):
        wide = torch.full((t.shape[0] + 1, t.shape[1] + 128), 0x7F, dtype=torch.uint8, device="cuda")
        wide[1:, 16:16 + t.shape[1]] = t
        return wide[1:, 16:16 + t.shape[1]]
    return ftm.ActCodes.of(inside(c.codes), inside(c.scales), c.rows, c.cols)


def one_of_two(c):
    """Only the codes as a view, of e4m3fn type."""
    return ftm.ActCodes.of(c.codes.t().contiguous().t().view(torch.float8_e4m3fn), c.scales, c.rows, c.cols)


VIEWS = (transposed, sliced, one_of_two)
SHAPES = ((16, 16), (48, 144), (128, 256), (384, 128), (272, 384))   # N, K: whole blocks of 128, and not


@pytest.mark.parametrize("view", VIEWS)
@pytest.mark.parametrize("N,K", SHAPES)
@pytest.mark.parametrize("T", (1, 128, 300))
def test_dense_weight_gradient(T, N, K, view):
    r = rng(T, N, K, 31)
    dy, x = form_of(matrix(r, T, N, spread=1)[0].T)[0], form_of(matrix(r, T, K, spread=1)[0].T)[0]
    a, b = view(dy), view(x)
    assert not a.codes.is_contiguous() or min(a.codes.shape) == 1
    want, got = torch.empty(N, K, device="cuda"), torch.empty(N, K, device="cuda")
    ftm.ft_linear_weight_grad(N, K, T, dy, x, want)
    ftm.ft_linear_weight_grad(N, K, T, a, b, got)
    assert torch.equal(want, got)
    ftm.ft_linear_weight_grad(N, K, T, a, x, got, accumulate=True)
    assert torch.equal(2 * want, got)


def experts_case(N, K):
    r = rng(N, K, 32)
    T, E, k = 200, 5, 2
    d, want, s = layout(r, T, E, k, 128)
    real = (want["row_pair"] >= 0)[:, None]
    dy, x = (form_of((matrix(r, d["rows"], C, spread=1)[0] * real).T)[0] for C in (N, K))
    return T, E, d, s, dy, x


@pytest.mark.parametrize("view", VIEWS)
@pytest.mark.parametrize("N,K", SHAPES)
def test_weight_gradients_of_experts(N, K, view):
    T, E, d, s, dy, x = experts_case(N, K)
    for kind in (torch.bfloat16, torch.float32):
        want, got = (torch.empty(E, N, K, dtype=kind, device="cuda") for _ in range(2))
        ftm.ft_expert_weight_grad(d, N, K, dy, x, s, T, want)
        for a, b in ((view(dy), view(x)), (view(dy), x), (dy, view(x))):
            ftm.ft_expert_weight_grad(d, N, K, a, b, s, T, got.fill_(7.0))
            assert torch.equal(want, got)


@pytest.mark.parametrize("R,K", ((2048, 2048), (2176, 2048), (128, 65536), (4112, 2048)))
def test_copies_of_large_views(R, K):
    """Four megabytes and more go through the weight transpose where their sizes allow it."""
    g = torch.Generator(device="cuda").manual_seed(R)
    v = torch.randint(0, 256, (K, R), generator=g, device="cuda", dtype=torch.uint8).t()
    c = ftm._laid_out(ftm.ActCodes.of(v, torch.zeros(K // 128, (R + 127) // 128 * 128, dtype=torch.uint8, device="cuda"), R, K), None)
    assert c.codes.is_contiguous() and torch.equal(c.codes, v)


def test_on_another_stream_and_captured():
    """The copies live on the call's stream: behind work that is still to fill the views, and in a replayed graph."""
    N, K = 128, 256
    T, E, d, s, dy, x = experts_case(N, K)
    want = torch.empty(E, N, K, device="cuda")
    ftm.ft_expert_weight_grad(d, N, K, dy, x, s, T, want)
    a, b, kept = transposed(dy), transposed(x), dy.codes.clone()
    other = torch.randint_like(kept, 0, 0x70)
    got, side = torch.empty_like(want), torch.cuda.Stream()
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        with torch.cuda.stream(side):
            a.codes.zero_()
            got.fill_(7.0)
            busy = torch.randn(2048, 2048, device="cuda")
            for _ in range(20):
                busy = busy @ busy * 1e-3
            a.codes.copy_(kept)
        ftm.ft_expert_weight_grad(d, N, K, a, b, s, T, got, stream=handle)
        side.synchronize()
        assert torch.equal(want, got)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ftm.ft_expert_weight_grad(d, N, K, a, b, s, T, got)
    for codes in (kept, other, kept):
        a.codes.copy_(codes)
        ftm.ft_expert_weight_grad(d, N, K, a, b, s, T, want)
        torch.cuda.synchronize()
        got.fill_(7.0)
        graph.replay()
        assert torch.equal(want, got)


def test_strided_outputs_and_other_shapes_are_refused():
    T, C = 128, 256
    x = torch.randn(T, C, device="cuda")
    with pytest.raises(ValueError, match="contiguous"):
        ftm.ft_act_quantize(x, T, C, col=transposed(ftm.ActCodes(C, T)))
    dy, dw = ftm.ActCodes(C, T), torch.empty(C, C, device="cuda")
    wrong = ftm.ActCodes.of(torch.zeros(T, 2 * C, dtype=torch.uint8, device="cuda")[:, ::2], dy.scales, C, T)
    with pytest.raises(ValueError, match="contiguous"):
        ftm.ft_linear_weight_grad(C, C, T, wrong, dy, dw)
    with pytest.raises(ValueError, match="contiguous"):
        ftm.ft_linear_weight_grad(C, C, T, dy, dy, torch.empty(C, C, device="cuda").t())
