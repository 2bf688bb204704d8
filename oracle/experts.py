"""Oracle of the routed experts in training and of the norms around a block: plain numpy in float64, TEST
INFRASTRUCTURE ONLY.

Written from the definitions, without the library's code: pairs sorted by expert, rows of tokens in that order and back,
products over the groups with their gradients, the two norms with gates and residual scale and their gradient."""
from __future__ import annotations

import numpy as np


def sort(ids, first, local, align, rows, mask=None):
    """Tables of ids [T][k]: a dict of row_pair, pair_row [T][k], off, count, dropped."""
    T, k = ids.shape
    row_pair, pair_row = np.full(rows, -1), np.full((T, k), -1)
    off, count, dropped = [0], [], 0
    for e in range(first, first + local):
        n = 0
        for t in range(T):
            for j in range(k):
                if ids[t, j] != e or (mask is not None and not mask[t]):
                    continue
                if off[-1] + n < rows:
                    row_pair[off[-1] + n], pair_row[t, j] = t * k + j, off[-1] + n
                    n += 1
                else:
                    dropped += 1
        count.append(n)
        off.append(off[-1] + -(-n // align) * align)   # rows is a multiple of align
    return {"row_pair": row_pair, "pair_row": pair_row, "off": np.array(off), "count": np.array(count),
            "dropped": np.array([dropped])}


def gather(s, x, weights=None):
    """Rows [off[-1]][C] of the groups, padding included."""
    k = s["pair_row"].shape[1]
    out = np.zeros((s["off"][-1], x.shape[1]))
    for r in range(len(out)):
        p = s["row_pair"][r]
        if p >= 0:
            out[r] = x[p // k] * (1.0 if weights is None else weights[p // k, p % k])
    return out


def combine(s, rows, weights=None, base=None):
    """(y [T][C], sum of the magnitudes of its terms)."""
    T, k = s["pair_row"].shape
    y = np.zeros((T, rows.shape[1])) if base is None else base.astype(np.float64).copy()
    mag = np.abs(y)
    for t, j in np.ndindex(T, k):
        if s["pair_row"][t, j] >= 0:
            v = rows[s["pair_row"][t, j]] * (1.0 if weights is None else weights[t, j])
            y[t] += v
            mag[t] += np.abs(v)
    return y, mag


def gate_grad(s, rows, dy):
    """(d_weights [T][k], sum of the magnitudes of its terms)."""
    d = np.zeros(s["pair_row"].shape)
    mag = np.zeros_like(d)
    for t, j in np.ndindex(d.shape):
        if s["pair_row"][t, j] >= 0:
            v = rows[s["pair_row"][t, j]] * dy[t]
            d[t, j], mag[t, j] = v.sum(), np.abs(v).sum()
    return d, mag


def product(s, x, w):
    """(y, magnitudes) [off[-1]][N] of rows x and weights w [local][N][K]; zeros in the padding."""
    y = np.zeros((s["off"][-1], w.shape[1]))
    mag = np.zeros_like(y)
    for e, n in enumerate(s["count"]):
        r = slice(s["off"][e], s["off"][e] + n)
        y[r], mag[r] = x[r] @ w[e].T, np.abs(x[r]) @ np.abs(w[e]).T
    return y, mag


def weight_grad(s, dy, x):
    """(dw, magnitudes) [local][N][K] of rows dy and x."""
    r = [slice(o, o + n) for o, n in zip(s["off"], s["count"])]
    return (np.stack([dy[i].T @ x[i] for i in r]), np.stack([np.abs(dy[i]).T @ np.abs(x[i]) for i in r]))


def _rms(v, eps):
    return np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


def norm(x, b, pre, post, gate, token_gate, post_norm, eps, scale):
    """(r, n); b may be None."""
    r = x
    if b is not None:
        u = post * b / _rms(b, eps) if post_norm else b
        r = x + scale * gate * token_gate[:, None] * u
    return r, pre * r / _rms(r, eps)


def norm_grad(r, b, dr, dn, pre, post, gate, token_gate, post_norm, eps, scale):
    """dx, d_block, pre, post, gate, token_gate, and each one's sum of magnitudes under "mag"."""
    h = token_gate[:, None]
    rr = _rms(r, eps)
    g, rh = dn * pre, r / rr
    m = (g * rh).mean(axis=1, keepdims=True)
    d = dr + (g - rh * m) / rr
    dmag = np.abs(dr) + (np.abs(g) + np.abs(rh) * np.abs(g * rh).mean(axis=1, keepdims=True)) / rr
    out = {"dx": d, "pre": (dn * rh).sum(axis=0)}
    mag = {"dx": dmag, "pre": np.abs(dn * rh).sum(axis=0)}
    if b is not None:
        q, qmag = scale * gate * h * d, np.abs(scale * gate * h) * dmag
        u, db, dbmag = b, q, qmag
        if post_norm:
            rb = _rms(b, eps)
            bh = b / rb
            v, vmag = q * post, qmag * np.abs(post)
            u = post * bh
            db = (v - bh * (v * bh).mean(axis=1, keepdims=True)) / rb
            dbmag = (vmag + np.abs(bh) * (vmag * np.abs(bh)).mean(axis=1, keepdims=True)) / rb
            out["post"], mag["post"] = (q * bh).sum(axis=0), (qmag * np.abs(bh)).sum(axis=0)
        out["d_block"], mag["d_block"] = db, dbmag
        out["gate"], mag["gate"] = (scale * h * d * u).sum(axis=0), (np.abs(scale * h * u) * dmag).sum(axis=0)
        out["token_gate"], mag["token_gate"] = (scale * gate * d * u).sum(axis=1), (np.abs(scale * gate * u) * dmag).sum(axis=1)
    return {**out, "mag": mag}
