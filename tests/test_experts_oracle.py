"""The oracle of the routed experts in training and of the norms, pinned: the tables by hand, every gradient against
differences of the function it belongs to.  CPU only."""
import numpy as np
import pytest

from oracle import experts


def test_tables_by_hand():
    ids = np.array([[2, 0], [2, 3], [1, 2], [2, 2]])
    s = experts.sort(ids, 1, 2, 16, 48)
    assert list(s["off"]) == [0, 16, 32] and list(s["count"]) == [1, 5] and s["dropped"][0] == 0
    assert list(s["row_pair"][:2]) == [4, -1] and list(s["row_pair"][16:22]) == [0, 2, 5, 6, 7, -1]
    assert np.array_equal(s["pair_row"], [[16, -1], [17, -1], [0, 18], [19, 20]])
    assert np.all(s["row_pair"][32:] == -1)
    s = experts.sort(ids, 1, 2, 16, 48, mask=[1, 0, 1, 1])
    assert list(s["count"]) == [1, 4] and s["pair_row"][1, 0] == -1


def test_tables_past_the_capacity():
    ids = np.array([[1], [0], [1], [2], [0]] * 7)                    # 14, 14 and 7 pairs
    s = experts.sort(ids, 0, 3, 16, 32)
    assert list(s["count"]) == [14, 14, 0] and s["dropped"][0] == 7
    s = experts.sort(np.concatenate([ids] * 2), 0, 3, 16, 48)       # 28, 28 and 14
    assert list(s["count"]) == [28, 16, 0] and s["dropped"][0] == 12 + 14
    assert (s["pair_row"] >= 0).sum() == 44 and list(s["off"]) == [0, 32, 48, 48]


def _differences(f, x, h=1e-6):
    d = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[i] = h
        d[i] = (f(x + e) - f(x - e)) / (2 * h)
    return d


def test_row_gradients_against_differences():
    r = np.random.default_rng(1)
    T, k, C = 5, 3, 4
    ids = r.integers(0, 4, (T, k))
    s = experts.sort(ids, 0, 3, 16, 64)
    x, w, dy = r.normal(size=(T, C)), r.normal(size=(T, k)), r.normal(size=(T, C))
    rows = r.normal(size=(s["off"][-1], C))
    y = lambda rows=rows, w=w: (experts.combine(s, rows, w)[0] * dy).sum()
    real = s["row_pair"][:len(rows)] >= 0
    assert np.allclose(_differences(lambda v: y(rows=v), rows)[real], experts.gather(s, dy, w)[real], atol=1e-8)
    assert np.allclose(_differences(lambda v: y(w=v), w), experts.gate_grad(s, rows, dy)[0], atol=1e-8)
    d = r.normal(size=rows.shape)
    g = _differences(lambda v: (experts.gather(s, v) * d).sum(), x)
    assert np.allclose(g, experts.combine(s, d)[0], atol=1e-8)
    W, N = r.normal(size=(3, 2, C)), 2
    dp = r.normal(size=(len(rows), N))
    f = lambda rows=rows, W=W: (experts.product(s, rows, W)[0] * dp).sum()
    assert np.allclose(_differences(lambda v: f(W=v), W), experts.weight_grad(s, dp, rows)[0], atol=1e-8)
    assert np.allclose(_differences(lambda v: f(rows=v), rows), experts.product(s, dp, W.transpose(0, 2, 1))[0], atol=1e-8)


@pytest.mark.parametrize("post_norm", (0, 1))
def test_norm_gradient_against_differences(post_norm):
    r = np.random.default_rng(2)
    T, C, eps, scale = 3, 5, 1e-2, 0.7
    x, b = r.normal(size=(T, C)), r.normal(size=(T, C))
    p = {"pre": r.normal(size=C), "post": r.normal(size=C), "gate": r.normal(size=C), "token_gate": r.normal(size=T)}
    dr, dn = r.normal(size=(T, C)), r.normal(size=(T, C))

    def loss(x=x, b=b, **kw):
        rv, n = experts.norm(x, b, post_norm=post_norm, eps=eps, scale=scale, **{**p, **kw})
        return (rv * dr).sum() + (n * dn).sum()

    rv, _ = experts.norm(x, b, post_norm=post_norm, eps=eps, scale=scale, **p)
    d = experts.norm_grad(rv, b, dr, dn, post_norm=post_norm, eps=eps, scale=scale, **p)
    assert np.allclose(_differences(lambda v: loss(x=v), x), d["dx"], atol=1e-7)
    assert np.allclose(_differences(lambda v: loss(b=v), b), d["d_block"], atol=1e-7)
    for n in ("pre", "gate", "token_gate") + (("post",) if post_norm else ()):
        assert np.allclose(_differences(lambda v: loss(**{n: v}), p[n]), d[n], atol=1e-7), n
    assert all(np.all(d["mag"][n] >= np.abs(d[n]) * (1 - 1e-12)) for n in d["mag"])
