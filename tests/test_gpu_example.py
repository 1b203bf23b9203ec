"""The scoring example end to end: training raises the tokens' log
probability, its gradient is torch's, and the 4-bit weights score nearly as the
full ones do."""

import os
import sys

import pytest

from gpu_util import note, torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, os.path.join(ROOT, "examples"))

pytestmark = pytest.mark.gpu


def test_score_tokens():
    import score_tokens as ex
    t = torch()
    note("examples/score_tokens.py")
    r = ex.main(["--vocab", "1001", "--dim", "100", "--rows", "500", "--steps", "30"])
    h = r["history"]
    assert h[0] == pytest.approx(-t.log(t.tensor(1001.0)).item(), abs=1e-4)   # uniform at first
    assert h[-1] > h[0] + 0.5 and all(b > a for a, b in zip(h[:5], h[1:6]))
    # the row alone gives the row's alternatives in the batch
    assert r["one"][3][0].tolist() == r["four"][3][0].tolist()
    # 4 bits lose some of what was learnt, not most of it
    assert r["four"][0] - h[0] > 0.5 * (r["full"][0] - h[0])
    assert r["agree"] > 0.3


def test_one_step_is_autograds():
    import score_tokens as ex
    t = torch()
    note("one training step against autograd")
    x, y = ex.data(64, 333, 48, 3, t.device("cuda"))
    w = t.randn((333, 48), device="cuda") * 0.1
    ref = w.clone().double().requires_grad_()
    lsm = t.log_softmax(x.double() @ ref.t(), 1)
    given = y >= 0
    lp = lsm.gather(1, y.clamp(min=0)[:, None])[:, 0][given].mean()
    ent = -(lsm.exp() * lsm).sum(1)[given].mean()
    (-lp - 0.01 * ent).backward()
    before = w.clone()
    ex.train(w, x, y, 1, lr=1.0, entropy_weight=0.01)
    step = (before - w).double()
    # fp32 products of 64 rows: a few ulps of the gradient's terms
    assert (step - ref.grad).abs().max() < 1e-6
