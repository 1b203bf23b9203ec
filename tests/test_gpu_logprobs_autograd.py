"""token_logprobs under autograd: outputs that depend on logits which require a
gradient carry one, and it is the gradient from the logits alone.

Tolerances as for the gradient of shifted logits: with u = 2^-24, p is off by
(V/256 + 72 + 3 |x - lse|) u of itself (the sums' terms, exp2, the differences),
H by (V/256 + 64) u (1 + H), an element's own n + 2 gradients by u each; bf16
rounds to 8 bits."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from oracle import logprobs as olp
from gpu_util import note, torch

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24


def _leaf(T, V, dtype, seed, shift=0.0):
    t = torch()
    x = (np.random.default_rng(seed).standard_normal((T, V)) * 3.0 + shift).astype(np.float32)
    return t.from_numpy(x).cuda().to(t.float32 if dtype == "f32" else t.bfloat16).requires_grad_()


def _tokens(T, V, seed):
    r = np.random.default_rng(seed)
    return np.where(r.random(T) < 0.8, r.integers(0, V, T), -1)


@pytest.mark.parametrize("T,V,n", [(5, 300, 0), (5, 300, 4), (1027, 2050, 3), (2, 20001, 20)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("parts", ["lp", "h", "lse", "top", "all"])
def test_backward(parts, dtype, T, V, n):
    t = torch()
    note(f"autograd of {parts} {dtype} T={T} V={V} n={n}")
    x = _leaf(T, V, dtype, V + n, 50.0)
    y = _tokens(T, V, 1)
    lp, h, lse, top, idx = pk.token_logprobs(x, t.from_numpy(y).cuda(), n)
    assert lp.requires_grad and h.requires_grad and lse.requires_grad and top.requires_grad and not idx.requires_grad
    r = np.random.default_rng(2)
    on = lambda part: parts in (part, "all")
    gl, gh, gz = (r.standard_normal(T).astype(np.float32) * on(p) for p in ("lp", "h", "lse"))
    gt = r.standard_normal((T, n)).astype(np.float32) * on("top")
    dev = lambda a: t.from_numpy(a).cuda()
    loss = 0.0
    if on("lp"):
        loss = loss + (lp * dev(gl)).sum()
    if on("h"):
        loss = loss + (h * dev(gh)).sum()
    if on("lse"):
        loss = loss + (lse * dev(gz)).sum()
    if on("top"):
        loss = loss + (top * dev(gt)).sum()
    loss.backward()
    assert x.grad.dtype == x.dtype and x.grad.shape == x.shape
    got, v, idx = x.grad.double().cpu().numpy(), x.detach().double().cpu().numpy(), idx.cpu().numpy()
    terms = V / 256 + 64
    for k in range(T):
        a = [float(gl[k]), float(gh[k]), idx[k], gt[k].astype(np.float64), float(gz[k])]
        ref = olp.grad_of_logits(v[k], int(y[k]), *a)
        l = olp.log_softmax(v[k])
        p = np.exp(l)
        H = -(p * l).sum()
        size = np.abs(a[3]).sum() + abs(a[4]) + (abs(a[0]) if y[k] >= 0 else 0.0) + abs(a[1]) * (np.abs(l) + H + 1.0)
        scale = p * size * (terms + 8 + 3 * np.abs(l))
        if y[k] >= 0:
            scale[y[k]] += abs(a[0]) * (2 + n)
        for j, g in zip(idx[k], a[3]):
            scale[j] += abs(g) * (2 + n)
        tol = U24 * scale + 1e-36 + (2.0 ** -8 * np.abs(ref) if dtype == "bf16" else 0.0)
        err = np.abs(got[k] - ref)
        assert (err <= tol).all(), (k, err.max(), (err / tol).max())


def test_sums_and_strided_logits():
    """The gradient of a plain sum arrives as one number spread over the rows;
    logits that are a part of wider rows; tokens that are all given.  Elements
    of up to 1 off by fewer than 32 u."""
    t = torch()
    note("autograd of sums of strided logits")
    wide = _leaf(6, 1003, "f32", 3)
    y = t.arange(6, device="cuda") * 7
    lp, h, _, _, _ = pk.token_logprobs(wide[:, 1:1001], y)
    (lp.sum() - 0.5 * h.mean()).backward()
    ref = wide.detach().double().requires_grad_()
    l = t.log_softmax(ref[:, 1:1001], 1)
    (l.gather(1, y[:, None]).sum() + 0.5 * (l.exp() * l).sum(1).mean()).backward()
    assert (wide.grad.double() - ref.grad).abs().max() < 2e-6
    assert not wide.grad[:, 0].any() and not wide.grad[:, 1001:].any()


def test_masked_and_empty_rows():
    t = torch()
    note("autograd of masked rows")
    x = _leaf(3, 500, "f32", 4)
    with t.no_grad():
        x[0] = -np.inf
        x[1, ::2] = -np.inf
    y = t.tensor([3, 5, -1], device="cuda")
    lp, h, lse, top, _ = pk.token_logprobs(x, y, 2)
    (lp[1:].sum() + h.sum() + lse[1:].sum() + top[1:].sum()).backward()
    g = x.grad
    assert t.isfinite(g).all() and not g[0].any() and not g[1, ::2].any()
    # a shift of a row moves its lse by as much, and nothing else
    assert abs(g[1].double().sum().item() - 1.0) < 1e-5 and abs(g[2].double().sum().item() - 1.0) < 1e-5


def test_what_is_recorded():
    t = torch()
    note("what autograd records")
    x, y = _leaf(4, 100, "f32", 5), t.zeros(4, dtype=t.int64, device="cuda")
    plain = pk.token_logprobs(x.detach(), y, 3)
    assert not any(o.requires_grad for o in plain)
    low, low_plain = t.full((4,), 7.0, device="cuda"), t.full((4,), 7.0, device="cuda")
    pk.token_logprobs(x.detach(), y, 3, lse_low=low_plain)
    for a, b in zip(plain, pk.token_logprobs(x, y, 3, lse_low=low)):
        assert t.equal(a, b)
    assert t.equal(low, low_plain)
    with t.no_grad():
        assert not any(o.requires_grad for o in pk.token_logprobs(x, y, 3))
    out = pk.token_logprobs_outputs(4, 3)
    assert pk.token_logprobs(x, y, 3, out=out) is out and not any(o.requires_grad for o in out)
    # logits changed between the two passes are torch's error, not a wrong gradient
    lp = pk.token_logprobs(x, y)[0]
    with t.no_grad():
        x.add_(1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        lp.sum().backward()
    for call in (lambda: pk.token_logprobs(x, y[:3]), lambda: pk.token_logprobs(x, y, 65),
                 lambda: pk.token_logprobs(x, y, lse_low=low[:2])):
        with pytest.raises(pk.ProfkError):
            call()
    with pytest.raises(pk.ProfkError, match="g_lse"):
        pk.token_logprobs_grad(x.detach(), y, low, low, low, g_lse=low[:3])


def test_a_training_step():
    """A step of an unembedding through the differentiable call, against torch's
    log_softmax in 64 bits."""
    t = torch()
    note("a training step under autograd")
    g = t.Generator(device="cuda").manual_seed(0)
    x = t.randn((64, 48), generator=g, device="cuda")
    w = (t.randn((333, 48), generator=g, device="cuda") * 0.1).requires_grad_()
    y = t.randint(333, (64,), generator=g, device="cuda")
    lp, h, lse, _, _ = pk.token_logprobs(x @ w.t(), y)
    (-lp.mean() - 0.01 * h.mean() + 1e-3 * (lse ** 2).mean()).backward()
    ref = w.detach().double().requires_grad_()
    z = x.double() @ ref.t()
    l = t.log_softmax(z, 1)
    (-l.gather(1, y[:, None]).mean() + 0.01 * (l.exp() * l).sum(1).mean()
     + 1e-3 * (t.logsumexp(z, 1) ** 2).mean()).backward()
    # fp32 products of 64 rows: a few ulps of the gradient's terms
    assert (w.grad.double() - ref.grad).abs().max() < 1e-6
