"""The gradient from the logits alone against differences and under shifts."""

import numpy as np
import pytest

from oracle import logprobs as olp


@pytest.mark.parametrize("y,top", [(3, []), (3, [3, 0, 0]), (-1, [1, 2]), (0, [-1, 50])])
def test_gradient_of_logits_equals_differences(y, top):
    g = np.random.default_rng(17)
    x = g.standard_normal(9) * 2
    g_lp, g_h, g_top = 0.7, -0.4, g.standard_normal(len(top))

    def f(z):
        lp, h, lse, _, _ = olp.row(z, y, 0)
        return g_lp * lp + g_h * h + sum(t * (z[j] - lse) for j, t in zip(top, g_top) if 0 <= j < z.size)

    d = olp.grad_of_logits(x, y, g_lp, g_h, top, g_top)
    assert np.abs(olp.grad_of_logits(x, y, g_lp, g_h, top, g_top, 0.3) - d - 0.3 * np.exp(olp.log_softmax(x))).max() < 1e-12
    e = 1e-5
    num = np.array([(f(x + e * np.eye(9)[j]) - f(x - e * np.eye(9)[j])) / (2 * e) for j in range(9)])
    assert np.abs(d - num).max() < 1e-9
    _, h, lse, _, _ = olp.row(x, y, 0)
    assert np.abs(d - olp.grad_row(x, y, lse, h, g_lp, g_h, top, g_top)).max() < 1e-12


@pytest.mark.parametrize("shift", [2.0 ** 10, -2.0 ** 13, 2.0 ** 20])
def test_gradient_of_logits_does_not_see_a_shift(shift):
    g = np.random.default_rng(18)
    x = np.round(g.standard_normal(50) * 3 * 2.0 ** 20) / 2.0 ** 20      # (exact with the shift)
    a = (7, 0.7, -0.4, [1, 2], [0.5, -0.25])
    d, e = olp.grad_of_logits(x, *a), olp.grad_of_logits(x + shift, *a)
    assert np.array_equal(d, e)
    assert d.sum() == pytest.approx(0.0, abs=1e-13)
