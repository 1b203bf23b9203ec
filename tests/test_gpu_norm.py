"""layer_norm and layer_norm_grad against their fp64 forms.

Tolerances, u = 2^-24: a row's or column's sum of n numbers is within (n_seq + 25)
u of the sum of their magnitudes, n_seq the longest run one thread adds (at most
16 in registers; D / 1024 rounded up to whole chunks of 8 for long rows).  Each
output adds half a step of its type, eps / 2 of itself."""

import numpy as np
import pytest
import torch

import paper_2608_12573_amd as pk
from oracle import dense
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _half(t):
    return torch.finfo(t).eps / 2


def _np(t):
    return t.detach().double().cpu().numpy()


def _inputs(T, D, dtype, seed, pad=0, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, D + pad), generator=g)
    x[:, ::61] *= 8.0
    x = x * torch.exp(0.5 * torch.randn((T, 1), generator=g)) + mean * torch.randn((T, 1), generator=g)
    w = 1.0 + 0.2 * torch.randn(D, generator=g)
    b = 0.1 * torch.randn(D, generator=g)
    return x.to(DT[dtype]).cuda()[:, :D], w, b


def _seq(D):
    return 16 if D <= 16384 else 8 * -(-D // 8192)


def _check(got, want, tol, what):
    err = np.abs(_np(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.2f} of the tolerance"


def _forward_tol(x, y, w, b, r, dtype):
    D = x.shape[1]
    s = (_seq(D) + 25) * U
    n = np.abs(x - x.mean(axis=1, keepdims=True)) * r[:, None]
    dm = s * np.abs(x).mean(axis=1, keepdims=True)                      # of the mean
    # of r: half the variance's, which sums squares (three roundings each); a few more for the root
    dr = 0.5 * (s + 4 * U) + 6 * U + (dm * r[:, None]) ** 2
    return np.abs(w) * (r[:, None] * dm + n * (dr + 4 * U)) + 2 * U * np.abs(b) + (_half(dtype) + 2 * U) * np.abs(y) + 1e-38


SHAPES = [(1, 1), (3, 2), (5, 7), (1, 4096), (4, 511), (9, 512), (7, 513), (5, 1000), (6, 1024), (3, 1025), (5, 2048), (3, 2049),
          (4, 4096), (3, 4097), (3, 6144), (2, 6145), (2, 8192), (3, 8193), (2, 12288), (3, 12289), (2, 16384), (3, 16385), (2, 50001), (2100, 96), (1500, 1536), (37, 777)]


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("xt,yt,wt", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"),
                                      ("bf16", "f32", "bf16")])
def test_forward(T, D, xt, yt, wt):
    note(f"layer_norm {T}x{D} {xt}->{yt} params {wt}")
    x, w, b = _inputs(T, D, xt, T * 7 + D, pad=T % 4)
    w, b = w.to(DT[wt]).cuda(), b.to(DT[wt]).cuda()
    y, m, r = pk.layer_norm(x, w, b, dtype=DT[yt])
    X, W, B = _np(x), _np(w), _np(b)
    ey, em, er = dense.layer_norm(X, W, B)
    assert y.dtype is DT[yt] and y.shape == (T, D)
    _check(m, em, (_seq(D) + 27) * U * np.abs(X).mean(axis=1) + 1e-38, "mean")
    _check(r, er, er * (0.5 * (_seq(D) + 29) * U + 8 * U + ((_seq(D) + 27) * U * np.abs(X).mean(axis=1) * er) ** 2), "rstd")
    _check(y, ey, _forward_tol(X, ey, W, B, er, DT[yt]), "out")


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("xt,yt,wt", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"),
                                      ("bf16", "f32", "f32")])
def test_grad(T, D, xt, yt, wt):
    note(f"layer_norm_grad {T}x{D} {xt} dy {yt} params {wt}")
    x, w, b = _inputs(T, D, xt, T * 5 + D)
    w = w.to(DT[wt]).cuda()
    dy = torch.randn((T, D + T % 3), generator=torch.Generator().manual_seed(T + D)).to(DT[yt]).cuda()[:, :D]
    _, m, r = pk.layer_norm(x, w)
    dx, dw, db = pk.layer_norm_grad(dy, x, w, m, r)
    assert dx.dtype is x.dtype and dw.dtype is w.dtype and db.dtype is w.dtype
    X, W, G, M, R = _np(x), _np(w), _np(dy), _np(m), _np(r)
    ex, ew, eb = dense.layer_norm_grad(G, X, W, M, R)
    s = (_seq(D) + 25) * U
    n, g = np.abs((X - M[:, None]) * R[:, None]), np.abs(G * W)
    gm, gn = g.mean(axis=1, keepdims=True), (g * n).mean(axis=1, keepdims=True)
    tol = np.abs(R[:, None]) * (6 * U * g + (s + 6 * U) * gm + n * (s + 12 * U) * gn) + _half(x.dtype) * np.abs(ex) + 1e-38
    _check(dx, ex, tol, "dx")
    # (at most all rows one after the other, and the parts)
    cols = (T + 30) * U
    _check(dw, ew, cols * (np.abs(G) * n).sum(axis=0) + _half(w.dtype) * np.abs(ew) + 1e-38, "dweight")
    _check(db, eb, cols * np.abs(G).sum(axis=0) + _half(w.dtype) * np.abs(eb) + 1e-38, "dbias")


def test_rows_far_from_zero_and_equal_rows():
    note("layer_norm of shifted and constant rows")
    g = torch.Generator().manual_seed(3)
    x = (torch.randn((6, 1000), generator=g) + 1e4).cuda()
    x[2] = 5.0
    x[4] = 0.0
    y, m, r = pk.layer_norm(x, None, None)
    ey, em, er = dense.layer_norm(_np(x))
    one = np.ones(1000)
    _check(y, ey, _forward_tol(_np(x), ey, one, 0 * one, er, torch.float32), "out")
    assert torch.isfinite(y).all()
    # rows of equal values: the mean's rounding, at most a few of its last bits,
    # is taken out again but for its own rounding, and rstd is 1 / sqrt(eps)
    for v in (5.0, 0.1, -1e4, 12345.678):
        z, mz, rz = pk.layer_norm(torch.full((2, 777), v, device="cuda"))
        assert z.abs().max() <= 2 * 45 * U * (45 * U * abs(v)) * 1e-5 ** -0.5 and (rz - 1e-5 ** -0.5).abs().max() <= 1e-3
        assert (mz - v).abs().max() <= 2 * U * abs(v)


@pytest.mark.parametrize("D", [100, 3000, 20000])
def test_nan_and_infinite_rows_stay_in_their_rows(D):
    note(f"layer_norm with NaN and inf, D {D}")
    x, w, b = _inputs(5, D, "f32", 4)
    x[1, D // 2] = float("nan")
    x[3, D - 1] = float("inf")
    y, m, r = pk.layer_norm(x, w.cuda(), b.cuda())
    assert torch.isnan(y[[1, 3]]).all() and torch.isfinite(y[[0, 2, 4]]).all()
    dx, dw, db = pk.layer_norm_grad(torch.ones_like(x), x, w.cuda(), m, r)
    assert torch.isnan(dx[[1, 3]]).all() and torch.isfinite(dx[[0, 2, 4]]).all()
    assert torch.isnan(dw).all() and torch.isfinite(db).all()


@pytest.mark.parametrize("D", [64, 1500, 9001, 17000])
def test_in_place_strides_and_neighbours(D):
    note(f"layer_norm in place and strided, D {D}")
    x, w, b = _inputs(6, D, "bf16", 5)
    w, b = w.cuda(), b.cuda()
    want = pk.layer_norm(x, w, b)
    big = torch.full((6, D + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    view = big[:, 3:3 + D]
    view.copy_(x)
    out = pk.layer_norm(view, w, b, out=(view, want[1].clone(), want[2].clone()))
    assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1]) and torch.equal(out[2], want[2])
    assert (big[:, :3] == 7).all() and (big[:, 3 + D:] == 7).all()
    # the gradient into a strided dx; rows and columns around it as they were
    dy = torch.randn((6, D), device="cuda").bfloat16()
    ref = pk.layer_norm_grad(dy, x, w, want[1], want[2])
    big.fill_(7.0)
    got = pk.layer_norm_grad(dy, x, w, want[1], want[2], out=(view, torch.empty_like(w), torch.empty_like(w)))
    for a, c in zip(got, ref):
        assert torch.equal(a, c)
    assert (big[:, :3] == 7).all() and (big[:, 3 + D:] == 7).all()


def test_rows_of_zero_and_parts_left_out():
    note("layer_norm without rows")
    w = torch.ones(33, device="cuda")
    x = torch.empty((0, 33), device="cuda")
    y, m, r = pk.layer_norm(x, w)
    dx, dw, db = pk.layer_norm_grad(x, x, w, m, r)
    assert y.shape == (0, 33) and (dw == 0).all() and (db == 0).all()
    x, w, _ = _inputs(40, 300, "f32", 8)
    w = w.cuda()
    _, m, r = pk.layer_norm(x, w)
    full = pk.layer_norm_grad(x, x, w, m, r)
    for need in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        part = pk.layer_norm_grad(x, x, w, m, r, need=need)
        for p, f, k in zip(part, full, need):
            assert torch.equal(p, f) if k else p is None


@pytest.mark.parametrize("T,D", [(3000, 200), (700, 5000), (600, 30000)])
def test_repeats_are_bitwise_equal(T, D):
    note(f"layer_norm_grad twice {T}x{D}")
    x, w, _ = _inputs(T, D, "bf16", 9)
    w = w.cuda()
    dy = torch.randn((T, D), device="cuda").bfloat16()
    _, m, r = pk.layer_norm(x, w)
    one, two = pk.layer_norm_grad(dy, x, w, m, r), pk.layer_norm_grad(dy, x, w, m, r)
    for a, c in zip(one, two):
        assert torch.equal(a, c)


@pytest.mark.parametrize("wt", ["f32", "bf16"])
def test_autograd(wt):
    note(f"layer_norm autograd {wt}")
    x, w, b = _inputs(20, 130, "f32", 10)
    x = x.contiguous().requires_grad_()
    w, b = w.to(DT[wt]).cuda().requires_grad_(), b.to(DT[wt]).cuda().requires_grad_()
    y, m, r = pk.layer_norm(x, w, b)
    assert y.requires_grad and not m.requires_grad
    d = torch.randn((20, 130), device="cuda")
    y.backward(d)
    want = pk.layer_norm_grad(d, x.detach(), w.detach(), m, r)
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[1]) and torch.equal(b.grad, want[2])
    # a sum's gradient is one number for all
    x2 = x.detach().clone().requires_grad_()
    pk.layer_norm(x2, None, b)[0].sum().backward()
    ref = pk.layer_norm_grad(torch.ones_like(d), x.detach(), None, m, r)
    assert torch.equal(x2.grad, ref[0])


def test_autograd_against_differences():
    note("layer_norm gradient against differences")
    x, w, b = _inputs(2, 9, "f32", 11)
    d = np.random.default_rng(0).normal(size=(2, 9))
    _, m, r = pk.layer_norm(x, w.cuda(), b.cuda())
    dx = _np(pk.layer_norm_grad(torch.tensor(d, dtype=torch.float32, device="cuda"), x, w.cuda(), m, r)[0])
    X, W, h = _np(x), _np(w), 1e-5
    for i in np.ndindex(2, 9):
        p, q = X.copy(), X.copy()
        p[i] += h
        q[i] -= h
        diff = ((dense.layer_norm(p, W)[0] - dense.layer_norm(q, W)[0]) * d).sum() / (2 * h)
        assert abs(diff - dx[i]) <= 1e-4 * (1 + abs(diff))
