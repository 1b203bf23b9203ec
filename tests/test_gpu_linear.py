"""linear and linear_grad against their fp64 forms.

Tolerances, u = 2^-24: a sum of K exact products is within (K + 2) u of the sum
of their magnitudes.  The activations have slopes of at most 1.13 and are
computed to 2^-20 of themselves plus 2^-22 absolutely, their slopes to 2^-20
absolutely; each output adds half a step of its type, eps / 2 of itself.  dz is
rounded to bf16, half a step of each of its terms."""

import numpy as np
import pytest
import torch

import paper_2608_12573_amd as pk
from oracle import dense
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
BF = torch.finfo(torch.bfloat16).eps / 2


def _half(t):
    return torch.finfo(t).eps / 2


def _np(t):
    return t.detach().double().cpu().numpy()


def _check(got, want, tol, what):
    err = np.abs(_np(got) - want)
    bad = ~(err <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, worst {np.nanmax(err / np.maximum(tol, 1e-300)):.2f} of the tolerance"


def _inputs(M, K, N, seed, pad=0, off=0):
    """x and w as views `off` elements into rows `pad` elements longer."""
    g = torch.Generator().manual_seed(seed)

    def rows(R, scale):
        t = torch.randn((R, K), generator=g) * scale
        big = torch.full((R, K + pad + off), 99.0, dtype=torch.bfloat16)
        big[:, off:off + K] = t.bfloat16()
        return big.cuda()[:, off:off + K]

    x, w = rows(M, 1.0), rows(N, K ** -0.5)
    return x, w, 0.5 * torch.randn(N, generator=g).cuda(), g


def _linear(M, K, N, act, out, bias, residual, seed, pad=0, off=0, pre=True):
    x, w, b, g = _inputs(M, K, N, seed, pad, off)
    b = b if bias else None
    r = torch.randn((M, N + pad), generator=g).to(DT[out]).cuda()[:, :N] if residual else None
    z = torch.empty((M, N), dtype=DT[out], device="cuda") if pre else None
    y = pk.linear(x, w, b, act, r, dtype=DT[out], pre=z)
    X, W = _np(x), _np(w)
    ey, ez = dense.linear(X, W, None if b is None else _np(b), act, None if r is None else _np(r))
    dz = (K + 3) * U * (np.abs(X) @ np.abs(W).T) + 2 * U * np.abs(ez)
    a = dense.act(ez, act)
    tol = 1.13 * dz + np.abs(a) * 2.0 ** -20 + 2.0 ** -22 + (_half(DT[out]) + U) * np.abs(ey)
    if pre:
        _check(z, ez, dz + (_half(DT[out]) + U) * np.abs(ez), "pre")
    assert y.dtype is DT[out] and y.shape == (M, N)
    _check(y, ey, tol, "out")
    return x, w, b, z


SHAPES = [(1, 1, 1), (1, 8, 1), (2, 3, 5), (1, 64, 100), (1, 4096, 1000), (3, 777, 130), (16, 512, 512), (17, 1000, 65),
          (32, 2048, 300), (33, 64, 33), (64, 72, 127), (100, 129, 257), (128, 128, 128), (127, 136, 255), (129, 64, 129),
          (256, 256, 256), (257, 200, 511), (300, 1001, 259), (512, 96, 640), (1000, 320, 777)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("act,out,bias,residual", [(None, "f32", False, False), ("gelu", "bf16", True, True),
                                                   ("silu", "f32", True, False), ("relu", "bf16", False, True)])
def test_forward(M, K, N, act, out, bias, residual):
    note(f"linear {M}x{K}x{N} {act} {out} bias {bias} residual {residual}")
    _linear(M, K, N, act, out, bias, residual, M + 3 * K + 7 * N)


# few rows: more groups of columns than are at work at once, with K shared by the
# waves of a workgroup or not; tiles of 256 x 256, and more than one a workgroup
@pytest.mark.parametrize("M,K,N", [(1, 72, 70000), (3, 584, 50008), (8, 512, 33000), (9, 64, 33001), (16, 1024, 9000),
                                   (17, 520, 33000), (32, 712, 5003), (1, 8192, 33), (5, 448, 140000), (31, 8, 100000),
                                   (4096, 64, 4096), (4000, 72, 4200), (5000, 136, 5003), (300, 8, 65541),
                                   (130, 200, 40000)])
@pytest.mark.parametrize("act,out", [(None, "f32"), ("gelu", "bf16")])
def test_many_groups_and_tiles(M, K, N, act, out):
    note(f"linear {M}x{K}x{N} {act} {out}")
    _linear(M, K, N, act, out, True, act is not None, M + K + N, pre=M < 1000)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 16])
@pytest.mark.parametrize("K,N", [(1, 3), (7, 100), (511, 65), (513, 1000), (1025, 33), (4097, 50), (101, 40003)])
@pytest.mark.parametrize("act,out,pad", [("gelu", "bf16", 0), (None, "f32", 1)])
def test_few_odd_rows(M, K, N, act, out, pad):
    note(f"linear {M}x{K}x{N} {act} {out} rows {pad} longer")
    _linear(M, K, N, act, out, True, act is not None, M + K + N, pad, pad)


@pytest.mark.parametrize("M,K,N", [(1, 4096, 640), (2, 72, 40), (9, 264, 96), (40, 1000, 200), (200, 264, 300), (300, 64, 520)])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (3, 2), (8, 0), (8, 8), (4, 4)])
def test_strides_and_alignment(M, K, N, pad, off):
    note(f"linear {M}x{K}x{N} rows {pad} longer, {off} in")
    _linear(M, K, N, "gelu", "bf16", True, True, M + K + N, pad, off)


def _grad(M, K, N, act, dt, seed, pad=0, off=0):
    x, w, b, g = _inputs(M, K, N, seed, pad, off)
    dy = torch.randn((M, N + pad), generator=g).to(DT[dt]).cuda()[:, :N]
    z = None
    if act:
        z = torch.empty((M, N), dtype=DT[dt], device="cuda")
        pk.linear(x, w, b, act, dtype=DT[dt], pre=z)
    dx, dw, db = pk.linear_grad(dy, x, w, z, act)
    X, W, G = _np(x), _np(w), _np(dy)
    ex, ew, eb, ez = dense.linear_grad(G, X, W, None if z is None else _np(z), act)
    off_z = 2.0 ** -20 * np.abs(G) + 2 * U * np.abs(ez)                    # the slope's and the product's
    t = BF * np.abs(ez) + off_z
    _check(dx, ex, t @ np.abs(W) + (N + 2) * U * (np.abs(ez) @ np.abs(W)) + BF * np.abs(ex) + 1e-38, "dx")
    _check(dw, ew, t.T @ np.abs(X) + (M + 2) * U * (np.abs(ez).T @ np.abs(X)) + BF * np.abs(ew) + 1e-38, "dw")
    _check(db, eb, off_z.sum(axis=0) + (M + 20) * U * np.abs(ez).sum(axis=0) + U * np.abs(eb) + 1e-38, "dbias")


@pytest.mark.parametrize("M,K,N", SHAPES + [(3000, 40, 72), (5000, 8, 16), (2048, 256, 256)])
@pytest.mark.parametrize("act,dt", [(None, "bf16"), (None, "f32"), ("gelu", "bf16"), ("silu", "f32"), ("relu", "bf16")])
def test_grad(M, K, N, act, dt):
    note(f"linear_grad {M}x{K}x{N} {act} {dt}")
    _grad(M, K, N, act, dt, M + K + N)


@pytest.mark.parametrize("M,K,N", [(8, 8, 8), (1500, 1000, 24), (24, 1500, 1000), (1000, 24, 1500), (1024, 1024, 1024),
                                   (2049, 1031, 515), (2304, 1032, 520), (3000, 2000, 128)])
@pytest.mark.parametrize("need", [(True, True, True), (True, True, False), (True, False, True), (False, True, True)])
def test_both_products_at_once_and_each_alone(M, K, N, need):
    note(f"linear_grad {M}x{K}x{N} {need}")
    x, w, b, g = _inputs(M, K, N, 12)
    dy = torch.randn((M, N), generator=g).bfloat16().cuda()
    got = pk.linear_grad(dy, x, w, need=need)
    X, W, G = _np(x), _np(w), _np(dy)
    ex, ew, eb, _ = dense.linear_grad(G, X, W, None)
    for t, want, tol in ((got[0], ex, (N + 2) * U * (np.abs(G) @ np.abs(W)) + BF * np.abs(ex) + 1e-38),
                         (got[1], ew, (M + 2) * U * (np.abs(G).T @ np.abs(X)) + BF * np.abs(ew) + 1e-38),
                         (got[2], eb, (M + 20) * U * np.abs(G).sum(axis=0) + U * np.abs(eb) + 1e-38)):
        if t is not None:
            _check(t, want, tol, "gradient")
    assert [t is not None for t in got] == list(need)


@pytest.mark.parametrize("M,K,N", [(4096, 4096, 64), (72, 4200, 4104), (4200, 72, 4104), (4100, 4360, 40)])
@pytest.mark.parametrize("act", [None, "gelu"])
def test_grad_of_large_tiles(M, K, N, act):
    note(f"linear_grad {M}x{K}x{N} {act}")
    _grad(M, K, N, act, "bf16", M + K + N)


@pytest.mark.parametrize("M,K,N", [(2, 72, 40), (64, 264, 96), (200, 264, 320), (300, 64, 520)])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (3, 2), (8, 0), (8, 8), (4, 4)])
@pytest.mark.parametrize("act", [None, "silu"])
def test_grad_strides_and_alignment(M, K, N, pad, off, act):
    note(f"linear_grad {M}x{K}x{N} {act} rows {pad} longer, {off} in")
    _grad(M, K, N, act, "bf16", M + K + N, pad, off)


@pytest.mark.parametrize("M,N", [(1, 40), (40, 300), (300, 520)])
def test_infinite_and_nan_rows(M, N):
    note(f"linear with infinities {M}x{N}")
    K = 64
    x, w, b, g = _inputs(M, K, N, 5)
    b[0], b[1], b[2] = float("inf"), -float("inf"), float("nan")
    for act in ("relu", "gelu", "silu"):
        z = torch.empty((M, N), device="cuda")
        y = pk.linear(x, w, b, act, pre=z)
        assert (y[:, 0] == float("inf")).all() and (y[:, 1] == 0).all() and torch.isnan(y[:, 2]).all()
        assert torch.isfinite(y[:, 3:]).all()
        db = pk.linear_grad(torch.ones_like(y), x, w, z, act, need=(False, False, True))[2]
        assert db[0].item() == M and db[1].item() == 0


@pytest.mark.parametrize("M,K,N", [(1, 256, 64), (70, 256, 136), (300, 512, 264)])
def test_residual_in_place_and_neighbours(M, K, N):
    note(f"linear into its residual {M}x{K}x{N}")
    x, w, b, g = _inputs(M, K, N, 6)
    r = torch.randn((M, N), generator=g).bfloat16().cuda()
    want = pk.linear(x, w, b, "gelu", r, dtype=torch.bfloat16)
    buf = torch.full((M * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[32:32 + M * N].view(M, N)
    out.copy_(r)
    pk.linear(x, w, b, "gelu", out, out=out)
    assert torch.equal(out, want) and (buf[:32] == 7).all() and (buf[32 + M * N:] == 7).all()


@pytest.mark.parametrize("M,K,N", [(2, 256, 65), (70, 256, 133), (300, 512, 261), (64, 4096, 515)])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
def test_outputs_at_any_element(M, K, N, dt):
    note(f"linear to odd places {M}x{K}x{N} {dt}")
    x, w, b, g = _inputs(M, K, N, 16)
    z = torch.empty((M, N), dtype=DT[dt], device="cuda")
    want = pk.linear(x, w, b, "silu", dtype=DT[dt], pre=z)
    bufs = [torch.full((M * N + 16,), 7.0, dtype=DT[dt], device="cuda") for _ in range(2)]
    out, pre = (t[3:3 + M * N].view(M, N) for t in bufs)
    pk.linear(x, w, b, "silu", out=out, pre=pre)
    assert torch.equal(out, want) and torch.equal(pre, z)
    for t in bufs:
        assert (t[:3] == 7).all() and (t[3 + M * N:] == 7).all()
    dy = torch.randn((M, N), generator=g).to(DT[dt]).cuda()
    grads = pk.linear_grad(dy, x, w, z, "silu")
    outs = [torch.full((t.numel() + 16,), 7.0, dtype=t.dtype, device="cuda") for t in grads]
    views = tuple(o[5:5 + t.numel()].view(t.shape) for o, t in zip(outs, grads))
    pk.linear_grad(dy, x, w, pre, "silu", out=views)
    for v, t, o in zip(views, grads, outs):
        assert torch.equal(v, t) and (o[:5] == 7).all() and (o[5 + t.numel():] == 7).all()


@pytest.mark.parametrize("N,parts", [(70000, "many columns"), (1100000, "more than one launch's")])
def test_wide_bias_gradients(N, parts):
    note(f"linear_grad of {N} columns")
    dy = torch.randn((3, N), generator=torch.Generator().manual_seed(N)).cuda()
    x = torch.ones((3, 8), dtype=torch.bfloat16, device="cuda")
    w = torch.ones((N, 8), dtype=torch.bfloat16, device="cuda")
    db = pk.linear_grad(dy, x, w, need=(False, False, True))[2]
    want = _np(dy).sum(axis=0)
    _check(db, want, 23 * U * np.abs(_np(dy)).sum(axis=0) + U * np.abs(want), "dbias")


def test_no_rows_no_columns():
    note("linear without rows or columns")
    w = torch.ones((5, 8), dtype=torch.bfloat16, device="cuda")
    x = torch.ones((3, 8), dtype=torch.bfloat16, device="cuda")
    assert pk.linear(x[:0], w).shape == (0, 5) and pk.linear(x, w[:0]).shape == (3, 0)
    dx, dw, db = pk.linear_grad(torch.empty((0, 5), device="cuda"), x[:0], w)
    assert dx.shape == (0, 8) and (dw == 0).all() and (db == 0).all()
    dx, dw, db = pk.linear_grad(torch.empty((3, 0), device="cuda"), x, w[:0])
    assert (dx == 0).all() and dw.shape == (0, 8) and db.shape == (0,)


@pytest.mark.parametrize("M,K,N", [(70, 264, 136), (600, 96, 80)])
@pytest.mark.parametrize("act", [None, "gelu"])
def test_parts_left_out_and_repeats(M, K, N, act):
    note(f"linear_grad parts {M}x{K}x{N} {act}")
    x, w, b, g = _inputs(M, K, N, 7)
    dy = torch.randn((M, N), generator=g).bfloat16().cuda()
    z = torch.empty_like(dy)
    pk.linear(x, w, b, act, pre=z, dtype=torch.bfloat16)
    full = pk.linear_grad(dy, x, w, z, act)
    for need in ((True, True, True), (True, False, False), (False, True, False), (False, False, True)):
        for p, f, k in zip(pk.linear_grad(dy, x, w, z, act, need=need), full, need):
            assert torch.equal(p, f) if k else p is None


@pytest.mark.parametrize("act", [None, "silu"])
def test_autograd(act):
    note(f"linear autograd {act}")
    x, w, b, g = _inputs(33, 72, 40, 8)
    r = torch.randn((33, 40), generator=g).cuda()
    leaves = [t.clone().requires_grad_() for t in (x, w, b, r)]
    y = pk.linear(*leaves[:3], activation=act, residual=leaves[3])
    d = torch.randn((33, 40), generator=g).cuda()
    y.backward(d)
    z = torch.empty((33, 40), device="cuda")
    pk.linear(x, w, b, act, pre=z)
    for leaf, want in zip(leaves, pk.linear_grad(d, x, w, z, act) + (d,)):
        assert torch.equal(leaf.grad, want)


def test_gradient_against_differences():
    note("linear gradient against differences")
    x, w, b, g = _inputs(2, 8, 3, 9)
    d = torch.randn((2, 3), generator=g).cuda()
    z = torch.empty((2, 3), device="cuda")
    pk.linear(x, w, b, "gelu", pre=z)
    dx, dw, db = (_np(t) for t in pk.linear_grad(d, x, w, z, "gelu"))
    X, W, B, G, h = _np(x), _np(w), _np(b), _np(d), 1e-5
    for got, at in ((dx, 0), (dw, 1), (db, 2)):
        for i in np.ndindex(*got.shape):
            p, q = [X.copy(), W.copy(), B.copy()], [X.copy(), W.copy(), B.copy()]
            p[at][i] += h
            q[at][i] -= h
            diff = ((dense.linear(*p, "gelu")[0] - dense.linear(*q, "gelu")[0]) * G).sum() / (2 * h)
            # dz and the result in bf16: two half steps of terms of up to 3 in size
            assert abs(diff - got[i]) <= 2 * BF * 6 + 1e-4
