"""The fp64 forms of layer norm, dense product and adjusted logits: against
differences, and at the ends of their ranges."""

import numpy as np
import pytest

from oracle import dense


def _diff(f, x, d, h=1e-6):
    """sum d * f's gradient by central differences, for each element of x."""
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        p, q = x.copy(), x.copy()
        p[i] += h
        q[i] -= h
        out[i] = ((f(p) - f(q)) * d).sum() / (2 * h)
    return out


def test_layer_norm_gradients():
    g = np.random.default_rng(0)
    x, w, b, d = g.normal(size=(3, 7)), g.normal(size=7), g.normal(size=7), g.normal(size=(3, 7))
    y, m, r = dense.layer_norm(x, w, b)
    np.testing.assert_allclose(((y - b) / w).mean(axis=1), 0, atol=1e-12)
    dx, dw, db = dense.layer_norm_grad(d, x, w, m, r)
    np.testing.assert_allclose(dx, _diff(lambda t: dense.layer_norm(t, w, b)[0], x, d), atol=1e-7)
    np.testing.assert_allclose(dw, _diff(lambda t: dense.layer_norm(x, t, b)[0], w, d), atol=1e-7)
    np.testing.assert_allclose(db, _diff(lambda t: dense.layer_norm(x, w, t)[0], b, d), atol=1e-7)


@pytest.mark.parametrize("act", [None, "relu", "gelu", "silu"])
def test_linear_gradients(act):
    g = np.random.default_rng(1)
    x, w, b, d = g.normal(size=(3, 5)), g.normal(size=(4, 5)), g.normal(size=4), g.normal(size=(3, 4))
    _, z = dense.linear(x, w, b, act)
    dx, dw, db, _ = dense.linear_grad(d, x, w, z, act)
    np.testing.assert_allclose(dx, _diff(lambda t: dense.linear(t, w, b, act)[0], x, d), atol=1e-7)
    np.testing.assert_allclose(dw, _diff(lambda t: dense.linear(x, t, b, act)[0], w, d), atol=1e-7)
    np.testing.assert_allclose(db, _diff(lambda t: dense.linear(x, w, t, act)[0], b, d), atol=1e-7)


def test_activation_limits():
    z = np.array([-np.inf, -200.0, 0.0, 200.0, np.inf])
    for name in ("relu", "gelu", "silu"):
        np.testing.assert_allclose(dense.act(z, name), [0, 0, 0, 200.0, np.inf], atol=1e-30)
        s = dense.slope(z, name)
        np.testing.assert_allclose(s[[0, 1, 3, 4]], [0, 0, 1, 1], atol=1e-30)


def test_adjust_by_hand():
    x = np.array([[2.0, -2.0, 0.0, 1.0, 3.0]])
    y = dense.adjust(x, [0, 1, 1, 7, -1, 3], [0, 6], [2], [2.0], [0.5], [0.25], ([3, 4, 3], [9.0, 1.0, -1.0], [0, 3]),
                     [[0b11011]], None)
    # 0 in the prompt alone; 1 there and once after it; 3 once after it, its last bias -1
    np.testing.assert_allclose(y, [[1.0, -4.75, -np.inf, 0.5 - 0.75 - 1.0, 4.0]])
    d = dense.adjust_grad(np.ones((1, 5)), x, [0, 1, 1, 3], [0, 4], [2.0], [[0b11011]], None)
    np.testing.assert_allclose(d, [[0.5, 2.0, 0.0, 0.5, 1.0]])
    assert np.isnan(dense.adjust(x, allowed=[[1]], mask=[1])).all()
    assert (dense.adjust(x, allowed=[[0]], mask=[-1]) == x).all()


def test_adjust_gradient():
    g = np.random.default_rng(2)
    x, d = g.normal(size=(2, 6)) * 2, g.normal(size=(2, 6))
    kw = dict(tokens=[1, 1, 4, 5, 0], offsets=[0, 3, 5], repetition=[1.5, 0.7], allowed=[[0b111011]])
    ok = np.isfinite(dense.adjust(x, **kw))
    f = lambda t: np.where(ok, dense.adjust(t, **kw), 0.0)   # noqa: E731
    np.testing.assert_allclose(dense.adjust_grad(d, x, **kw), _diff(f, x, d), atol=1e-7)
