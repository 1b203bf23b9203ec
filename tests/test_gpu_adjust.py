"""adjust_logits and adjust_logits_grad against their fp64 forms.

Tolerances, u = 2^-24: the logit's penalty is rounded once, the product of count
and frequency, the sum of both penalties, the difference and the bias once each:
4 u of each magnitude that enters, and half a step of the output."""

import numpy as np
import pytest
import torch

import paper_2608_12573_amd as pk
from oracle import dense
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
INF = float("inf")


def _np(t):
    return None if t is None else t.detach().cpu().numpy() if t.dtype in (torch.int32, torch.int64) else t.double().cpu().numpy()


def _case(T, V, dtype, seed, history=40, masks=2, biases=6, pad=0, prompt=True):
    g = torch.Generator().manual_seed(seed)
    x = (3 * torch.randn((T, V + pad), generator=g)).to(DT[dtype]).cuda()[:, :V]
    n = torch.randint(0, history + 1, (T,), generator=g)
    n[::4] = 0
    at = torch.zeros(T + 1, dtype=torch.int64)
    at[1:] = n.cumsum(0)
    tokens = torch.randint(-1, V + 1, (int(at[-1]),), generator=g)          # (some are none)
    tokens[::3] = tokens[::3] % 5
    kw = dict(tokens=tokens, offsets=at, n_prompt=n // 2 if prompt else None, repetition=0.5 + torch.rand(T, generator=g),
              presence=torch.rand(T, generator=g) - 0.3, frequency=torch.rand(T, generator=g) - 0.3)
    if biases:
        m = torch.randint(0, biases + 1, (T,), generator=g)
        bat = torch.zeros(T + 1, dtype=torch.int64)
        bat[1:] = m.cumsum(0)
        ids = torch.randint(-1, V + 1, (int(bat[-1]),), generator=g)
        ids[::2] = ids[::2] % 3                                             # (repeated ones)
        kw["bias"] = (ids, 4 * torch.randn(len(ids), generator=g), bat)
    if masks:
        kw["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (masks, -(-V // 32)), generator=g).to(torch.int32)
        kw["mask"] = torch.randint(-1, masks, (T,), generator=g)
    return x, {k: tuple(t.cuda() for t in v) if k == "bias" else None if v is None else v.cuda() for k, v in kw.items()}


def _want(x, kw):
    host = {k: tuple(_np(t) for t in v) if k == "bias" else _np(v) for k, v in kw.items()}
    X = _np(x)
    with np.errstate(invalid="ignore", over="ignore"):
        y = dense.adjust(X, **host)
        c = np.zeros_like(X)
        rep = host.get("repetition")
        size = np.abs(X) * (1 if rep is None else np.maximum(rep, 1 / rep)[:, None])
        for r in range(X.shape[0]):
            made, _ = dense._row(r, X.shape[1], host.get("tokens"), host.get("offsets"), host.get("n_prompt"))
            c[r] = made
        for name, k in (("presence", c > 0), ("frequency", c)):
            if host.get(name) is not None:
                size = size + k * np.abs(host[name])[:, None]
        if host.get("bias") is not None and len(host["bias"][1]):
            size = size + np.abs(host["bias"][1]).max()
    return y, 4 * U * size


def _check(y, want, tol, dtype):
    got = _np(y)
    nan = np.isnan(want)
    assert (np.isnan(got) == nan).all() and (np.isposinf(got) == np.isposinf(want)).all() and \
        (np.isneginf(got) == np.isneginf(want)).all()
    ok = np.isfinite(want)
    err = np.abs(got[ok] - want[ok])
    lim = tol[ok] + (torch.finfo(DT[dtype]).eps / 2) * np.abs(want[ok]) + 1e-38
    assert (err <= lim).all(), f"worst {np.max(err / lim):.2f} of the tolerance"


SHAPES = [(1, 1), (3, 2), (2, 31), (2, 32), (5, 33), (4, 100), (7, 1000), (1, 1024), (2, 1025), (3, 4100), (1, 8193),
          (2, 50001), (600, 65), (300, 2051), (40, 20000)]


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masks,biases,prompt", [(2, 6, True), (0, 0, False)])
def test_forward(T, V, dtype, masks, biases, prompt):
    note(f"adjust_logits {T}x{V} {dtype} masks {masks} biases {biases}")
    x, kw = _case(T, V, dtype, T + V, masks=masks, biases=biases, pad=T % 3, prompt=prompt)
    y = pk.adjust_logits(x, **kw)
    assert y.dtype is x.dtype
    _check(y, *_want(x, kw), dtype)


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masks", [0, 3])
def test_grad(T, V, dtype, masks):
    note(f"adjust_logits_grad {T}x{V} {dtype} masks {masks}")
    x, kw = _case(T, V, dtype, T * 3 + V, masks=masks, biases=0, pad=T % 3)
    d = torch.randn((T, V + 1), generator=torch.Generator().manual_seed(V)).to(DT[dtype]).cuda()[:, :V]
    kw = {k: kw.get(k) for k in ("tokens", "offsets", "repetition", "allowed", "mask")}
    y = pk.adjust_logits_grad(d, x, **kw)
    want = dense.adjust_grad(_np(d), _np(x), **{k: _np(v) for k, v in kw.items()})
    _check(y, want, 2 * U * np.abs(want), dtype)


@pytest.mark.parametrize("history", [1, 2, 513, 5000])
@pytest.mark.parametrize("V", [40, 3000, 30000])
def test_histories(history, V):
    note(f"adjust_logits history {history} of {V}")
    x, kw = _case(5, V, "f32", history + V, history=history, masks=0, biases=0)
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), "f32")
    # one token over and over
    one = dict(kw, tokens=torch.full_like(kw["tokens"], V - 1))
    _check(pk.adjust_logits(x, **one), *_want(x, one), "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [33, 5000, 40001])
def test_histories_past_the_small_counts(V, dtype):
    note(f"adjust_logits long histories of {V} {dtype}")
    x, kw = _case(6, V, dtype, V, history=50000, masks=2, biases=400)
    n = (kw["offsets"][1:] - kw["offsets"][:-1]).tolist()
    assert max(n) > 16384 and any(0 < k < 16384 for k in n)
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), dtype)
    # 16383 times, 16384 times and more, one token
    at = torch.tensor([0, 16383, 16383 + 16384, 16383 + 16384 + 16385, 60000, 60000, 60001], device="cuda")
    one = dict(kw, tokens=torch.full((60001,), V - 1, device="cuda"), offsets=at, n_prompt=None)
    _check(pk.adjust_logits(x, **one), *_want(x, one), dtype)
    g = {k: one[k] for k in ("tokens", "offsets", "repetition", "allowed", "mask")}
    d = torch.randn((6, V), device="cuda").to(DT[dtype])
    want = dense.adjust_grad(_np(d), _np(x), **{k: _np(v) for k, v in g.items()})
    _check(pk.adjust_logits_grad(d, x, **g), want, 2 * U * np.abs(want), dtype)


@pytest.mark.parametrize("V,n", [(40, 300), (3000, 900), (30000, 3000)])
def test_many_biases(V, n):
    note(f"adjust_logits {n} biases of {V}")
    x, kw = _case(4, V, "f32", n, biases=n)
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), "f32")
    # all of them on few tokens
    few = dict(kw, bias=(kw["bias"][0] % 7,) + kw["bias"][1:])
    _check(pk.adjust_logits(x, **few), *_want(x, few), "f32")


@pytest.mark.parametrize("V", [1, 31, 64, 130, 256, 700, 3000, 9000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_token_marked(V, dtype):
    note(f"adjust_logits every token of {V} marked {dtype}")
    x, kw = _case(5, V, dtype, V, masks=2, biases=40)
    every = torch.arange(V, device="cuda")
    kw["tokens"] = torch.cat([every, every.flip(0)[:V // 2]]).repeat(5)
    kw["offsets"] = torch.arange(6, device="cuda") * (V + V // 2)
    kw["n_prompt"] = torch.tensor([0, V // 3, V, 10 * V, 1], device="cuda")
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), dtype)


@pytest.mark.parametrize("name", ["repetition", "presence", "frequency", "bias", "allowed", None])
def test_each_alone(name):
    note(f"adjust_logits with {name} alone")
    x, kw = _case(6, 500, "bf16", 3)
    keep = {"bias": ["bias"], "allowed": ["allowed", "mask"], None: []}.get(name, ["tokens", "offsets", name])
    kw = {k: v for k, v in kw.items() if k in keep}
    y = pk.adjust_logits(x, **kw)
    _check(y, *_want(x, kw), "bf16")
    if name is None:
        assert torch.equal(y, x)


def test_masks_by_row_and_for_all():
    note("adjust_logits masks without row numbers")
    x, kw = _case(3, 200, "f32", 4, masks=3)
    kw.pop("mask")
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), "f32")
    kw["allowed"] = kw["allowed"][:1].contiguous()
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), "f32")
    # one that allows nothing, none, and one that is not there
    kw["allowed"] = torch.zeros_like(kw["allowed"])
    kw["mask"] = torch.tensor([0, -5, 1], device="cuda")
    y = pk.adjust_logits(x, **kw)
    assert (y[0] == -INF).all() and torch.isfinite(y[1]).all() and torch.isnan(y[2]).all()
    d = pk.adjust_logits_grad(torch.ones_like(x), x, kw["tokens"], kw["offsets"], None, kw["repetition"], kw["allowed"], kw["mask"])
    assert (d[0] == 0).all() and torch.isfinite(d[1]).all() and torch.isnan(d[2]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_infinities_and_lowest_values(dtype):
    note(f"adjust_logits unusual logits {dtype}")
    x, kw = _case(8, 300, dtype, 5)
    low = torch.finfo(DT[dtype]).min
    for v, col in ((float("nan"), 0), (INF, 1), (-INF, 2), (low, 3), (-low, 4), (0.0, 0), (-0.0, 1)):
        x[:, col + 5 * (v == 0)] = v
    kw["repetition"].clamp_(min=1.0)
    kw["repetition"][2] = 1.0
    y, (want, tol) = pk.adjust_logits(x, **kw), _want(x, kw)
    with np.errstate(over="ignore"):       # (what leaves the type's range is infinite)
        top = float(torch.finfo(DT[dtype]).max)
        over = np.isfinite(want) & (np.abs(want) > top)
        want = np.where(over, np.sign(want) * INF, want)
    _check(y, want, tol, dtype)


def test_lists_that_point_outside():
    note("adjust_logits offsets outside the lists")
    x, kw = _case(4, 100, "f32", 6, masks=0)
    n, m = len(kw["tokens"]), len(kw["bias"][0])
    kw["offsets"] = torch.tensor([-7, 3, n + 50, 2, 2 ** 40], device="cuda")
    kw["n_prompt"] = torch.tensor([100, -3, 2, 1], device="cuda")
    kw["bias"] = kw["bias"][:2] + (torch.tensor([0, m + 9, 1, -4, m], device="cuda"),)
    host = {k: tuple(_np(t) for t in v) if k == "bias" else _np(v) for k, v in kw.items()}
    host["bias"] = (host["bias"][0], host["bias"][1], np.clip(host["bias"][2], 0, m))
    want = dense.adjust(_np(x), **host)
    _check(pk.adjust_logits(x, **kw), want, 4 * U * (np.abs(_np(x)) * 2 + 100), "f32")


@pytest.mark.parametrize("T,V", [(3, 1000), (2, 20001)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_neighbours(T, V, dtype):
    note(f"adjust_logits in place {T}x{V} {dtype}")
    x, kw = _case(T, V, dtype, 7)
    want = pk.adjust_logits(x, **kw)
    big = torch.full((T, V + 9), 7.0, dtype=DT[dtype], device="cuda")
    view = big[:, 5:5 + V]
    view.copy_(x)
    pk.adjust_logits(view, out=view, **kw)
    assert torch.equal(view, want) and (big[:, :5] == 7).all() and (big[:, 5 + V:] == 7).all()
    g = {k: kw[k] for k in ("tokens", "offsets", "repetition", "allowed", "mask")}
    d = torch.randn((T, V), device="cuda").to(DT[dtype])
    want = pk.adjust_logits_grad(d, x, **g)
    view.copy_(d)
    pk.adjust_logits_grad(view, x, out=view, **g)
    assert torch.equal(view, want) and (big[:, :5] == 7).all() and (big[:, 5 + V:] == 7).all()
    big.fill_(7.0)
    pk.adjust_logits(x, out=view, **kw)
    assert (big[:, :5] == 7).all() and (big[:, 5 + V:] == 7).all()


def test_no_rows():
    note("adjust_logits without rows")
    x = torch.empty((0, 50), device="cuda")
    assert pk.adjust_logits(x).shape == (0, 50) and pk.adjust_logits_grad(x, x).shape == (0, 50)


def test_autograd():
    note("adjust_logits autograd")
    x, kw = _case(6, 400, "f32", 8)
    leaf = x.clone().requires_grad_()
    y = pk.adjust_logits(leaf, **kw)
    d = torch.randn((6, 400), device="cuda")
    y.backward(d)
    want = pk.adjust_logits_grad(d, x, kw["tokens"], kw["offsets"], None, kw["repetition"], kw["allowed"], kw["mask"])
    assert torch.equal(leaf.grad, want)
    # against differences, where nothing is forbidden and no logit near 0
    host = {k: tuple(_np(t) for t in v) if k == "bias" else _np(v) for k, v in kw.items()}
    X, G, W, h = _np(x), _np(d), _np(want), 1e-6
    for r, v in ((1, 3), (2, 4), (3, 100), (5, 399)):
        p, q = X.copy(), X.copy()
        p[r, v] += h
        q[r, v] -= h
        a, c = dense.adjust(p, **host)[r, v], dense.adjust(q, **host)[r, v]
        diff = 0.0 if np.isinf(a) else (a - c) / (2 * h) * G[r, v]
        assert abs(diff - W[r, v]) <= 1e-6 * (1 + abs(diff))
