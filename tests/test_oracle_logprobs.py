"""The log probability oracle against torch's log_softmax and against
differences, and its cases without a value of their own."""

import numpy as np
import pytest
import torch

from oracle import logprobs as olp


@pytest.mark.parametrize("V,seed", [(1, 0), (2, 1), (17, 2), (300, 3)])
def test_row_equals_log_softmax(V, seed):
    g = np.random.default_rng(seed)
    x = g.standard_normal(V) * 3
    n = min(V, 5)
    lp, h, lse, top, idx = olp.row(x, V - 1, n)
    ref = torch.log_softmax(torch.from_numpy(x), 0)
    assert lp == pytest.approx(ref[V - 1].item(), abs=1e-12)
    assert lse == pytest.approx(torch.logsumexp(torch.from_numpy(x), 0).item(), abs=1e-12)
    assert h == pytest.approx(-(ref.exp() * ref).sum().item(), abs=1e-12)
    v, i = torch.topk(ref, n)
    assert np.array_equal(idx, i.numpy()) and np.allclose(top, v.numpy(), atol=1e-12)


def test_ties_and_masks():
    x = np.array([1.0, -np.inf, 2.0, 2.0, -0.0, 0.0, -np.inf])
    _, _, _, top, idx = olp.row(x, 0, 7)
    assert idx.tolist() == [2, 3, 0, 5, 4, -1, -1]
    assert top[-1] == -np.inf and top[0] == top[1]


def test_rows_without_values():
    ninf = np.full(4, -np.inf)
    lp, h, lse, top, idx = olp.row(ninf, 2, 2)
    assert (lp, h, lse) == (-np.inf, 0.0, -np.inf) and idx.tolist() == [-1, -1]
    assert olp.row(ninf, -1, 0)[0] == 0.0
    for bad in (np.nan, np.inf):
        lp, h, lse, _, idx = olp.row(np.array([0.0, bad, 1.0]), 0, 1)
        assert np.isnan(lp) and np.isnan(h) and np.isnan(lse) and idx.tolist() == [1]
    assert np.isnan(olp.row(np.zeros(3), 3, 0)[0])
    low = np.full(8, float(np.finfo(np.float32).min))
    lp, h, _, _, _ = olp.row(low, 3, 0)
    assert lp == pytest.approx(-np.log(8)) and h == pytest.approx(np.log(8))
    assert not olp.grad_row(ninf, 0, -np.inf, 0.0, 1.0, 1.0, [], []).any()
    assert np.isnan(olp.grad_row(np.zeros(3), 5, np.log(3), np.log(3), 1.0, None, [], [])).all()


@pytest.mark.parametrize("y,top", [(3, []), (3, [3, 0, 0]), (-1, [1, 2]), (0, [-1, 50])])
def test_gradient_equals_differences(y, top):
    g = np.random.default_rng(7)
    x = g.standard_normal(9) * 2
    g_lp, g_h, g_top = 0.7, -0.4, g.standard_normal(len(top))

    def f(z):
        lp, h, lse, _, _ = olp.row(z, y, 0)
        return g_lp * lp + g_h * h + sum(t * (z[j] - lse) for j, t in zip(top, g_top) if 0 <= j < z.size)

    _, h, lse, _, _ = olp.row(x, y, 0)
    d = olp.grad_row(x, y, lse, h, g_lp, g_h, top, g_top)
    e = 1e-5
    num = np.array([(f(x + e * np.eye(9)[j]) - f(x - e * np.eye(9)[j])) / (2 * e) for j in range(9)])
    assert np.abs(d - num).max() < 1e-9
    assert d.sum() == pytest.approx(0.0, abs=1e-12)   # softmax does not see a shift


def test_gradient_of_masked_logits_is_zero_but_for_the_token():
    x = np.array([0.5, -np.inf, 1.0])
    _, h, lse, _, _ = olp.row(x, 0, 0)
    d = olp.grad_row(x, 1, lse, h, 2.0, 0.5, [], [])
    assert d[1] == 2.0
