"""Oracle of the dense 8-bit operators: plain numpy in float64, TEST INFRASTRUCTURE ONLY.

Written from the definitions, without the library's code: the 8-bit form of a matrix, the product over it
and its weight gradient, the SwiGLU between two products and its gradient, and the router's balance loss
with its gradient.  Matrices are float64 arrays; an 8-bit form is (codes uint8 [R][Kp], scale bytes
uint8 [Kp/128][R])."""
from __future__ import annotations

import numpy as np

from . import GATE_SOFTMAX, e4m3fn_value

_VALUES = np.array([e4m3fn_value(c) for c in range(256)])
_POSITIVE = _VALUES[:127]      # codes 0 .. 126 in ascending order of their values


def pad128(n: int) -> int:
    return -(-n // 128) * 128


def nearest_code(v: np.ndarray) -> np.ndarray:
    """e4m3fn code nearest to each v (|v| <= 448), ties to the even code; the sign bit is v's."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def scale_exponent(amax: np.ndarray) -> np.ndarray:
    """Smallest e in [-127, 127] with 448 * 2^e >= amax; 0 where amax is 0."""
    e = np.full(amax.shape, 127)
    for k in range(127, -128, -1):
        e = np.where(448.0 * 2.0 ** k >= amax, k, e)
    return np.where(amax == 0, 0, e)


def quantize(x: np.ndarray):
    """8-bit form of x [R][K]."""
    R, K = x.shape
    b = np.zeros((R, pad128(K)))
    b[:, :K] = x
    b = b.reshape(R, -1, 128)
    finite = np.isfinite(b)
    e = scale_exponent(np.abs(np.where(finite, b, 0.0)).max(axis=2))
    codes = nearest_code(np.where(finite, b, 0.0) * 2.0 ** -e[:, :, None].astype(float))
    codes = np.where(finite, codes, 0x7F).astype(np.uint8)
    return codes.reshape(R, -1), (e + 127).astype(np.uint8).T.copy()


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The matrix [R][Kp] an 8-bit form stands for."""
    return _VALUES[codes] * np.repeat(2.0 ** (scales[:, :codes.shape[0]].T.astype(float) - 127), 128, axis=1)


def weight_values(w: np.ndarray, s: np.ndarray) -> np.ndarray:
    """The weight [N][Kp] of codes w and block scales s."""
    n, k = np.arange(w.shape[0]) // 128, np.arange(w.shape[1]) // 128
    return _VALUES[w] * s.astype(np.float64)[n][:, k]


def sigmoid(z: np.ndarray) -> np.ndarray:
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def swiglu(gu: np.ndarray) -> np.ndarray:
    g, u = np.split(gu, 2, axis=1)
    return g * sigmoid(g) * u


def swiglu_grad(gu: np.ndarray, dh: np.ndarray) -> np.ndarray:
    g, u = np.split(gu, 2, axis=1)
    s = sigmoid(g)
    return np.concatenate([dh * u * s * (1 + g * (1 - s)), dh * g * s], axis=1)


def probabilities(logits: np.ndarray, gating: int) -> np.ndarray:
    """Router probabilities over all experts; zeros for a token whose logits are all -inf."""
    out = np.zeros_like(logits)
    for t, l in enumerate(logits):
        live = l > -np.inf
        if not live.any():
            continue
        v = l[live]
        # the sigmoids as exp(min(l, 0)) / (1 + exp(-|l|)), relative to the largest exp(min(l, 0))
        w = v - v.max() if gating == GATE_SOFTMAX else np.minimum(v, 0) - min(v.max(), 0) - np.log1p(np.exp(-np.abs(v)))
        w = np.exp(w)
        out[t, live] = w / w.sum()
    return out


def counted(T: int, seq_off, mask):
    """Counted tokens of each sequence."""
    live = np.ones(T, bool) if mask is None else np.asarray(mask) != 0
    return [np.arange(b, e)[live[b:e]] for b, e in zip(seq_off[:-1], seq_off[1:])]


def balance(logits, topk_ids, seq_off, mask, gating: int, coef: float):
    """dict of counts, tokens, prob, frac, loss per sequence."""
    T, E = logits.shape
    k = topk_ids.shape[1]
    p = probabilities(logits, gating)
    out = {n: [] for n in ("counts", "tokens", "prob", "frac", "loss")}
    for rows in counted(T, seq_off, mask):
        n = len(rows)
        ids = topk_ids[rows].ravel()
        c = np.bincount(ids[(ids >= 0) & (ids < E)], minlength=E)
        P = p[rows].sum(axis=0) / max(n, 1)
        f = coef * E * c / (k * max(n, 1))
        for name, v in zip(("counts", "tokens", "prob", "frac", "loss"), (c, n, P, f, (f * P).sum())):
            out[name].append(v)
    return {n: np.array(v) for n, v in out.items()}


def router_grad(logits, topk_ids, topk_w, d_topk_w, seq_off, mask, gating: int, frac, d_loss):
    """(d_logits, magnitude of its terms), rows of tokens in no sequence NaN; frac [n_seq][E] as given."""
    T, E = logits.shape
    p = probabilities(logits, gating)
    a = np.ones_like(logits) if gating == GATE_SOFTMAX else sigmoid(-logits)
    d, mag = np.full((T, E), np.nan), np.zeros((T, E))
    for s, (b, e) in enumerate(zip(seq_off[:-1], seq_off[1:])):
        d[b:e] = 0
        rows = counted(T, seq_off, mask)[s]
        if d_loss is not None and len(rows):
            w, dot = d_loss[s] / len(rows), p[rows] @ frac[s]
            d[rows] += w * p[rows] * a[rows] * (frac[s][None] - dot[:, None])
            mag[rows] += np.abs(w) * p[rows] * a[rows] * (np.abs(frac[s])[None] + np.abs(dot)[:, None])
        if d_topk_w is not None:
            for t in range(b, e):
                ids = topk_ids[t]
                ok = (ids >= 0) & (ids < E)
                dot = (topk_w[t] * d_topk_w[t])[ok].sum()
                for j in np.flatnonzero(ok):
                    q = topk_w[t, j] * a[t, ids[j]]
                    d[t, ids[j]] += q * (d_topk_w[t, j] - dot)
                    mag[t, ids[j]] += q * (abs(d_topk_w[t, j]) + np.abs(topk_w[t] * d_topk_w[t])[ok].sum())
    return d, mag
