"""Tensors of more than 2^32 elements: rows near the end of layer_norm, linear,
adjust_logits and their gradients are those of a call with these rows alone."""

import pytest
import torch

import paper_2608_12573_amd as pk
from gpu_util import note

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _room():
    yield
    torch.cuda.empty_cache()


def _rows(T, D, seed, dtype=torch.bfloat16):
    """T rows that repeat 1000 random ones, the last 40 of their own."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((T, D), dtype=dtype, device="cuda")
    base = torch.randn((1000, D), generator=g, device="cuda").to(dtype)
    for r in range(0, T, 1000):
        x[r:r + 1000] = base[:min(1000, T - r)]
    x[-40:] = torch.randn((40, D), generator=g, device="cuda").to(dtype)
    return x


def test_layer_norm():
    T, D = 530_000, 8192
    note(f"layer_norm {T}x{D}")
    x = _rows(T, D, 1)
    w, b = torch.rand(D, device="cuda"), torch.rand(D, device="cuda")
    y, m, r = pk.layer_norm(x, w, b)
    ty, tm, tr = pk.layer_norm(x[-40:].contiguous(), w, b)
    assert torch.equal(y[-40:], ty) and torch.equal(m[-40:], tm) and torch.equal(r[-40:], tr)
    assert torch.equal(y[:900], y[-1000:-100])
    dx = pk.layer_norm_grad(y, x, w, m, r, need=(True, False, False))[0]
    td = pk.layer_norm_grad(ty, x[-40:].contiguous(), w, tm, tr, need=(True, False, False))[0]
    assert torch.equal(dx[-40:], td)


def test_linear():
    M, K, N = 66_000, 8, 66_000
    note(f"linear {M}x{K}x{N}")
    x, w = _rows(M, K, 2), _rows(N, K, 3)
    bias = torch.rand(N, device="cuda")
    y = pk.linear(x, w, bias, "relu", dtype=torch.bfloat16)
    assert torch.equal(y[-40:], pk.linear(x[-40:].contiguous(), w, bias, "relu", dtype=torch.bfloat16))
    # as an operand: rows of dz past 2^32 elements
    dx, dw, db = pk.linear_grad(y, x, w, y, "relu")
    t = pk.linear_grad(y[-40:].contiguous(), x[-40:].contiguous(), w, y[-40:].contiguous(), "relu",
                       need=(True, False, False))[0]
    # (the same sums of 66000 products in other parts: 2 steps of the result, and 66002 u of the terms)
    size = y[-40:].double().abs() @ w.double().abs()
    assert ((dx[-40:].double() - t.double()).abs() <= 2.0 ** -7 * t.double().abs() + 66002 * 2.0 ** -23 * size).all()
    want = torch.zeros(N, dtype=torch.float64, device="cuda")
    for r in range(0, M, 6000):
        want += y[r:r + 6000].double().sum(dim=0)
    # (dz = y where z > 0: sums of positive numbers, (M + 20) u of themselves)
    assert ((db.double() - want).abs() <= (M + 20) * 2.0 ** -24 * want + 1e-30).all()


def test_adjust_logits():
    T, V = 34_000, 131_072
    note(f"adjust_logits {T}x{V}")
    x = _rows(T, V, 4)
    g = torch.Generator(device="cuda").manual_seed(5)
    tokens = torch.randint(V, (T * 10,), generator=g, device="cuda")
    at = torch.arange(T + 1, device="cuda") * 10
    rep = 1 + torch.rand(T, generator=g, device="cuda")
    allowed = torch.randint(-2 ** 31, 2 ** 31, (3, V // 32), generator=g, device="cuda").to(torch.int32)
    mask = torch.randint(-1, 3, (T,), generator=g, device="cuda")
    last = dict(tokens=tokens[-400:].contiguous(), offsets=at[:41].contiguous(), repetition=rep[-40:].contiguous(),
                allowed=allowed, mask=mask[-40:].contiguous())
    out = torch.empty_like(x)
    pk.adjust_logits(x, tokens, at, repetition=rep, allowed=allowed, mask=mask, out=out)
    assert torch.equal(out[-40:], pk.adjust_logits(x[-40:].contiguous(), **last))
    d = torch.ones_like(x)
    pk.adjust_logits_grad(d, x, tokens, at, repetition=rep, allowed=allowed, mask=mask, out=out)
    assert torch.equal(out[-40:], pk.adjust_logits_grad(d[-40:].contiguous(), x[-40:].contiguous(), **last))
