"""The gradient of shifted logits against the gradient from the logits alone.

Tolerance, with u = 2^-24: the forward pass's lse is off by (V/256 + 64) u (its
sums' terms, as in the forward tests), and so is each p of itself; x - lse, the
difference less lse_low and its product with log2 e are off by u |x - lse| each,
exp2 and a term's own products by 8 u.  H is off by (V/256 + 64) u (1 + H).  An
element's own gradients are added in fp32, n + 2 of them.  bf16 rounds the
result to 8 bits.  From an lse rounded to fp32 alone, p is off by u |lse| more."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from oracle import logprobs as olp
from gpu_util import note, torch

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24


def _logits(T, V, shift, dtype, seed):
    t = torch()
    x = (np.random.default_rng(seed).standard_normal((T, V)) * 3.0 + shift).astype(np.float32)
    g = t.from_numpy(x).cuda().to(t.float32 if dtype == "f32" else t.bfloat16)
    return g, g.double().cpu().numpy()


def _check(g, v, n, low, entropy):
    t = torch()
    T, V = g.shape
    r = np.random.default_rng(V)
    y = r.integers(0, V, T)
    y[r.random(T) < 0.2] = -1
    yd = t.from_numpy(y).cuda()
    lse_low = t.full((T,), 7.0, device="cuda") if low else None
    _, h, lse, _, idx = pk.token_logprobs(g, yd, n, lse_low=lse_low)
    gl, gt = r.standard_normal(T).astype(np.float32), r.standard_normal((T, n)).astype(np.float32)
    gh = r.standard_normal(T).astype(np.float32) if entropy else None
    dev = lambda a: t.from_numpy(a).cuda() if a is not None else None
    d = pk.token_logprobs_grad(g, yd, lse, h, dev(gl), dev(gh), idx if n else None, dev(gt) if n else None, lse_low=lse_low)
    got, idx, lse = d.double().cpu().numpy(), idx.cpu().numpy(), lse.double().cpu().numpy()
    terms = V / 256 + 64
    for k in range(T):
        top, g_h = gt[k].astype(np.float64), None if gh is None else float(gh[k])
        ref = olp.grad_of_logits(v[k], int(y[k]), float(gl[k]), g_h, idx[k], top)
        l = np.maximum(olp.log_softmax(v[k]), -1e4)
        p = np.exp(l)
        H = -(p * l).sum()
        total = (abs(gl[k]) if y[k] >= 0 else 0.0) + np.abs(top).sum()
        size = total + (abs(g_h) * (np.abs(l) + H + 1.0) if entropy else 0.0)
        scale = p * size * (terms + 8 + 3 * np.abs(l) + (0.0 if low else abs(lse[k])))
        if y[k] >= 0:
            scale[y[k]] += abs(gl[k]) * (2 + n)
        for j, a in zip(idx[k], top):
            scale[j] += abs(a) * (2 + n)
        tol = U24 * scale + 1e-36 + (2.0 ** -8 * np.abs(ref) if g.dtype == t.bfloat16 else 0.0)
        err = np.abs(got[k] - ref)
        assert (err <= tol).all(), (k, err.max(), (err / tol).max())


# one wave's rows; a workgroup's; rows split over workgroups, in several pieces
SHAPES = [(30, 300, 3), (30, 300, 0), (1027, 3001, 0), (3, 20001, 5)]


@pytest.mark.parametrize("T,V,n", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0.0, 1000.0, -1000.0, 9000.0, -15000.0, 30000.0, 1e6])
def test_shifted(shift, dtype, T, V, n):
    note(f"gradient of logits around {shift} {dtype} T={T} V={V} n={n}")
    g, v = _logits(T, V, shift, dtype, V)
    for entropy in (False, True):
        _check(g, v, n, True, entropy)


@pytest.mark.parametrize("shift", [1000.0, 9000.0])
def test_shifted_without_the_low_part(shift):
    """The bound that the header states for an lse that is rounded to fp32."""
    note(f"gradient of logits around {shift}, lse alone")
    g, v = _logits(30, 300, shift, "f32", 300)
    _check(g, v, 3, False, True)


def test_low_part():
    """lse + lse_low is the log-sum-exp; 0 where lse is not finite."""
    t = torch()
    low_value = float(np.finfo(np.float32).min)
    for T, V in ((7, 300), (7, 20001)):
        note(f"lse_low T={T} V={V}")
        g, _ = _logits(T, V, 5000.0, "f32", 3)
        g[1] = -np.inf
        g[2, 5] = np.nan
        g[3, 7] = np.inf
        g[4] = low_value
        g[5] *= 1e30
        y = t.zeros(T, dtype=t.int64, device="cuda")
        lse_low = t.full((T,), 7.0, device="cuda")
        plain = pk.token_logprobs(g, y, 4)
        out = pk.token_logprobs(g, y, 4, lse_low=lse_low)
        for a, b in zip(plain, out):
            assert np.array_equal(a.cpu().numpy(), b.cpu().numpy(), equal_nan=True)
        lse, low = out[2].double().cpu().numpy(), lse_low.double().cpu().numpy()
        assert not low[1:4].any()
        v = g.double().cpu().numpy()
        for r in (0, 4, 5, 6):
            m = v[r].max()
            err = ((lse[r] - m) + low[r]) - np.log(np.exp(v[r] - m).sum())
            assert abs(err) <= (V / 256 + 66) * U24
        # the gradient of a row of the lowest value: uniform
        one = t.ones(T, device="cuda")
        d = pk.token_logprobs_grad(g, y, out[2], out[1], one, lse_low=lse_low).double().cpu().numpy()
        assert not d[1].any() and np.isnan(d[2:4]).all()
        assert np.abs(d[4, 1:] + 1.0 / V).max() <= (V / 256 + 80) * U24 / V


def test_refusals():
    t = torch()
    x, y, f = t.zeros(4, 16, device="cuda"), t.zeros(4, dtype=t.int64, device="cuda"), t.zeros(4, device="cuda")
    for low in (f[:3], f.double(), f.cpu(), [0.0] * 4, t.zeros(8, device="cuda")[::2]):
        with pytest.raises(pk.ProfkError, match="lse_low"):
            pk.token_logprobs(x, y, lse_low=low)
        with pytest.raises(pk.ProfkError, match="lse_low"):
            pk.token_logprobs_grad(x, y, f, f, f, lse_low=low)
