"""The history encoder's oracle against closed forms and differences (CPU)."""

import numpy as np
import pytest

from oracle import encoder_oracle as enc

RNG = np.random.default_rng


def difference(f, x, step=1e-5):
    """Gradient of the scalar f at x by central differences."""
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        a, b = x.copy(), x.copy()
        a[i] += step
        b[i] -= step
        g[i] = (f(a) - f(b)) / (2 * step)
    return g


def test_rotation_keeps_lengths_and_depends_on_distance_alone():
    r = RNG(1)
    q, k = r.standard_normal((1, 1, 8)), r.standard_normal((1, 1, 8))
    at = lambda x, p: enc.norm_rotary(x, None, np.array([p]), 100.0, 0.0)[0][0, 0]  # noqa: E731
    assert np.linalg.norm(at(q, 37)) == pytest.approx(np.sqrt(8.0))
    assert at(q, 5) @ at(k, 2) == pytest.approx(at(q, 105) @ at(k, 102))
    assert np.allclose(at(q, 0), enc.norm_rotary(q, None, None, 100.0, 0.0)[0][0, 0])
    # the first pair turns by one radian a position
    y, z = at(q, 1), at(q, 0)
    assert y[0] == pytest.approx(z[0] * np.cos(1) - z[4] * np.sin(1)) and y[4] == pytest.approx(z[4] * np.cos(1) + z[0] * np.sin(1))


def test_rotary_gradients():
    r = RNG(2)
    x, gamma, dy, pos = r.standard_normal((3, 2, 6)), r.standard_normal(6), r.standard_normal((3, 2, 6)), np.array([0, 7, -3])
    (dx, dg), _ = enc.norm_rotary_backward(dy, x, gamma, pos, 50.0, 1e-3)
    f = lambda x, g: (enc.norm_rotary(x, g, pos, 50.0, 1e-3)[0] * dy).sum()  # noqa: E731
    assert np.allclose(dx, difference(lambda v: f(v, gamma), x), atol=1e-8)
    assert np.allclose(dg, difference(lambda v: f(x, v), gamma), atol=1e-8)


@pytest.mark.parametrize("causal", [True, False])
def test_attention_gradients(causal):
    r = RNG(3)
    qs, ks = enc.spans([0, 3, 5, 9], None, 9), enc.spans([0, 3, 8, 10], None, 10)  # equal, more keys, more queries than keys
    Q, K, V, dO = (r.standard_normal((n, h, 4)) for n, h in ((9, 4), (10, 2), (10, 2), (9, 4)))
    f = lambda q, k, v: (enc.sequence_attention(q, k, v, qs, ks, 0.7, causal)[0] * dO).sum()  # noqa: E731
    O, _, inside = enc.sequence_attention(Q, K, V, qs, ks, 0.7, causal)
    dQ, dK, dV = enc.sequence_attention_backward(dO, Q, K, V, O, inside, 0.7)
    assert np.allclose(dQ, difference(lambda x: f(x, K, V), Q), atol=1e-8)
    assert np.allclose(dK, difference(lambda x: f(Q, x, V), K), atol=1e-8)
    assert np.allclose(dV, difference(lambda x: f(Q, K, x), V), atol=1e-8)


def test_attention_is_the_framework_s_own_target_attention_without_a_mask():
    from oracle import lime_oracle as orc

    r = RNG(4)
    d, h = 8, 2
    T, E = r.standard_normal((1, 5, d)), r.standard_normal((1, 7, d))
    Wq, Wk, Wv = (r.standard_normal((d, d)) for _ in range(3))
    want = orc.mha_target_attention(T, E, np.array([7]), Wq, Wk, Wv, h, 0.5)[0]
    heads = lambda x: x.reshape(-1, h, d // h)  # noqa: E731
    got, _, _ = enc.sequence_attention(heads(T[0] @ Wq), heads(E[0] @ Wk), heads(E[0] @ Wv), [(0, 5, 5)], [(0, 7, 7)], 0.5, False)
    assert np.allclose(got.reshape(5, d), want)


def test_attention_row_by_row():
    """Causal, aligned at the end: the last query alone sees what it sees among the others; a query before all keys sees nothing."""
    r = RNG(5)
    Q, K, V = (r.standard_normal((6, 1, 4)) for _ in range(3))
    O, lse, _ = enc.sequence_attention(Q, K, V, [(0, 6, 6)], [(0, 6, 6)], 0.5, True)
    assert np.allclose(O[0], V[0]) and lse[0, 0] == pytest.approx(0.5 * Q[0, 0] @ K[0, 0])
    one, _, _ = enc.sequence_attention(Q[5:], K, V, [(0, 1, 1)], [(0, 6, 6)], 0.5, True)
    assert np.allclose(one[0], O[5])
    few, l, _ = enc.sequence_attention(Q, K[:2], V[:2], [(0, 6, 6)], [(0, 2, 2)], 0.5, True)
    assert (few[:4] == 0).all() and np.isneginf(l[:4]).all() and np.allclose(few[4], V[0])


def test_loss_and_gradients():
    r = RNG(6)
    X, W, t, dl = r.standard_normal((5, 3)), r.standard_normal((7, 3)), np.array([2, -1, 6, 2, 7]), r.standard_normal(5)
    loss, lse, _ = enc.catalogue_loss(X, W, t, 1.3)
    z = 1.3 * X[0] @ W.T
    assert loss[0] == pytest.approx(-np.log(np.exp(z[2]) / np.exp(z).sum())) and loss[1] == loss[4] == lse[1] == 0
    f = lambda x, w: (enc.catalogue_loss(x, w, t, 1.3)[0] * dl).sum()  # noqa: E731
    dX, dW = enc.catalogue_loss_backward(dl, X, W, t, 1.3)
    assert np.allclose(dX, difference(lambda v: f(v, W), X), atol=1e-8) and np.allclose(dW, difference(lambda v: f(X, v), W), atol=1e-8)
