"""The oracle of the dense 8-bit operators, pinned: its 8-bit form against a search over all codes and
torch's conversion, its gradients against differences of the losses they belong to.  CPU only."""
import numpy as np
import pytest
import torch

import oracle
from oracle import dense


def test_nearest_code_against_all_codes_and_torch():
    rng = np.random.default_rng(0)
    v = np.concatenate([rng.uniform(-448, 448, 400), rng.normal(0, 0.01, 400), dense._POSITIVE,
                        (dense._POSITIVE[1:] + dense._POSITIVE[:-1]) / 2, [0.0, -0.0, 448.0, -448.0]])
    v = v.astype(np.float32).astype(np.float64)
    c = dense.nearest_code(v)
    best = np.nanmin(np.abs(dense._VALUES[None] - v[:, None]), axis=1)
    assert np.array_equal(np.abs(dense._VALUES[c] - v), best)
    t = torch.from_numpy(v).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(c, t)


def test_scale_is_the_smallest_that_covers():
    amax = np.array([448.0, np.nextafter(448.0, 500), 449.0, 224.0, 1.0, 1.75, 1.7500001, 3e38, 1e-45, 448 * 2.0 ** -127])
    e = dense.scale_exponent(amax)
    assert np.all(448 * 2.0 ** e.astype(float) >= amax)
    inner = e > -127
    assert np.all(448 * 2.0 ** (e[inner].astype(float) - 1) < amax[inner])
    assert dense.scale_exponent(np.zeros(1))[0] == 0


def test_quantize_error_is_half_a_step_and_values_invert():
    rng = np.random.default_rng(1)
    x = rng.normal(size=(5, 300)) * 10.0 ** rng.integers(-6, 6, (5, 1))
    codes, scales = dense.quantize(x)
    assert codes.shape == (5, 384) and scales.shape == (3, 5) and not codes[:, 300:].any()
    v = dense.values(codes, scales)[:, :300]
    step = np.repeat(2.0 ** (scales.T.astype(float) - 127), 128, axis=1)[:, :300]
    assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step))
    again, s2 = dense.quantize(v)
    assert np.array_equal(again[:, :300], codes[:, :300]) and np.array_equal(s2, scales)


def test_swiglu_gradient_against_differences():
    rng = np.random.default_rng(2)
    gu, dh = rng.normal(size=(3, 8)) * 3, rng.normal(size=(3, 4))
    d = dense.swiglu_grad(gu, dh)
    for i in np.ndindex(gu.shape):
        h = 1e-6
        e = np.zeros_like(gu)
        e[i] = h
        num = ((dense.swiglu(gu + e) - dense.swiglu(gu - e)) * dh).sum() / (2 * h)
        assert abs(num - d[i]) < 1e-8


@pytest.mark.parametrize("gating", (oracle.GATE_SOFTMAX, oracle.GATE_SIGMOID))
def test_router_gradient_against_differences(gating):
    rng = np.random.default_rng(3)
    T, E, k, off = 7, 6, 2, [0, 3, 3, 6]
    logits = rng.normal(size=(T, E)) - (2 if gating else 0)
    mask = np.array([1, 0, 1, 1, 1, 1, 1])
    ids = np.argsort(-logits, axis=1)[:, :k]
    d_loss, dw = rng.normal(size=3), rng.normal(size=(T, k))

    def gates(l):
        sel = np.take_along_axis(l, ids, 1)
        v = np.exp(sel) if gating == oracle.GATE_SOFTMAX else dense.sigmoid(sel)
        return v / v.sum(axis=1, keepdims=True)

    def total(l):
        b = dense.balance(l, ids, off, mask, gating, 0.7)
        return (b["loss"] * d_loss).sum() + (gates(l) * dw)[:6].sum()

    b = dense.balance(logits, ids, off, mask, gating, 0.7)
    assert list(b["tokens"]) == [2, 0, 3] and not b["loss"][1] and not b["prob"][1].any()
    d, _ = dense.router_grad(logits, ids, gates(logits), dw, off, mask, gating, b["frac"], d_loss)
    assert np.isnan(d[6]).all()
    for i in np.ndindex(6, E):
        e = np.zeros_like(logits)
        e[i] = 1e-6
        assert abs((total(logits + e) - total(logits - e)) / 2e-6 - d[i]) < 1e-7


def test_probabilities_of_far_logits():
    l = np.array([[-200.0, -201.0, -np.inf], [-np.inf] * 3, [1.0, 500.0, -500.0]])
    p = dense.probabilities(l, oracle.GATE_SIGMOID)
    assert np.allclose(p[0], [1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1)), 0]) and not p[1].any()
    s = dense.sigmoid(l[2])
    assert np.allclose(p[2], s / s.sum())
