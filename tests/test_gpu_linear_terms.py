"""linear_grad's products take dz = dy act'(z) within 2^-16 of itself, not rounded to
bf16, where the caller does not ask for that.

Tolerances, u = 2^-24: the first of dz's two bf16 numbers is within 2^-8 of it, the
second within 2^-8 of what is left, 2^-16 of dz.  A sum of 2 N exact products, whose
terms' magnitudes are 1 + 2^-7 of the whole's at most, is within (2 N + 3) u of these
(1.01 of the whole's magnitudes).  Slopes are computed to 2^-20 absolutely; a result
is rounded once, eps / 2 of itself."""

import numpy as np
import pytest
import torch

import paper_2608_12573_amd as pk
from oracle import dense
from tests.gpu_util import note
from tests.test_gpu_linear import BF, DT, U, _check, _inputs, _np

pytestmark = pytest.mark.gpu
ONE = 2.0 ** -12


def _grad(M, K, N, act, dt, pad=0, off=0, need=(True, True, True)):
    x, w, b, g = _inputs(M, K, N, M + 5 * K + N, pad, off)
    dy = torch.randn((M, N + pad), generator=g).to(DT[dt]).cuda()[:, :N]
    z = None
    if act:
        z = torch.empty((M, N), dtype=DT[dt], device="cuda")
        pk.linear(x, w, b, act, dtype=DT[dt], pre=z)
    dx, dw, _ = pk.linear_grad(dy, x, w, z, act, need=need)
    X, W, G = _np(x), _np(w), _np(dy)
    ex, ew, _, ez = dense.linear_grad(G, X, W, None if z is None else _np(z), act)
    size = np.abs(ez)
    off_z = 2.0 ** -16 * size + (2.0 ** -20 * np.abs(G) if act else 0) + 2 * U * size
    if dx is not None:
        _check(dx, ex, off_z @ np.abs(W) + 1.01 * (2 * N + 3) * U * (size @ np.abs(W)) + BF * np.abs(ex) + 1e-38, "dx")
    if dw is not None:
        _check(dw, ew, off_z.T @ np.abs(X) + 1.01 * (2 * M + 3) * U * (size.T @ np.abs(X)) + BF * np.abs(ew) + 1e-38, "dw")


# (both products at once, each alone, tiles of either size, K in parts)
SHAPES = [(1, 1, 1), (2, 3, 5), (17, 100, 65), (33, 64, 33), (64, 72, 127), (64, 264, 64), (65, 72, 129), (127, 136, 255),
          (128, 128, 128), (257, 200, 511), (300, 1001, 259), (512, 96, 640), (1024, 24, 40), (40, 520, 1500)]


@pytest.mark.parametrize("M,K,N", SHAPES)
@pytest.mark.parametrize("act,dt", [(None, "f32"), ("gelu", "bf16"), ("silu", "f32"), ("relu", "bf16"), ("relu", "f32")])
def test_grad(M, K, N, act, dt):
    note(f"linear_grad in two terms {M}x{K}x{N} {act} {dt}")
    _grad(M, K, N, act, dt)


@pytest.mark.parametrize("M,K,N", [(4096, 4096, 40), (72, 4200, 1032), (4200, 1032, 72), (3000, 40, 72), (5000, 136, 16)])
@pytest.mark.parametrize("need", [(True, True, False), (True, False, False), (False, True, False)])
def test_large_tiles_and_parts(M, K, N, need):
    note(f"linear_grad in two terms {M}x{K}x{N} {need}")
    _grad(M, K, N, None, "f32", need=need)


@pytest.mark.parametrize("M,K,N", [(2, 72, 40), (64, 264, 96), (200, 264, 320)])
@pytest.mark.parametrize("pad,off", [(1, 0), (0, 1), (3, 2), (8, 8)])
@pytest.mark.parametrize("act,dt", [(None, "f32"), ("silu", "bf16")])
def test_strides_and_alignment(M, K, N, pad, off, act, dt):
    note(f"linear_grad in two terms {M}x{K}x{N} {act} {dt} rows {pad} longer, {off} in")
    _grad(M, K, N, act, dt, pad, off)


@pytest.mark.parametrize("M,K,N", [(1, 8, 2), (3, 8, 130), (130, 72, 64), (64, 264, 4096), (300, 1001, 258), (4096, 4096, 66)])
@pytest.mark.parametrize("off", [0, 1])
def test_what_bf16_would_lose(M, K, N, off):
    """Pairs of 1 + e and -1: only the e are left, multiples of 2^-12 whose sums are
    exact in fp32."""
    note(f"linear_grad of differences {M}x{K}x{N} {off} in")
    e = torch.randint(-7, 8, (M, N // 2), generator=torch.Generator().manual_seed(N)) * ONE
    dy = torch.empty((M, N))
    dy[:, ::2], dy[:, 1::2] = 1 + e, -1
    w = torch.ones((N, K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    x = torch.zeros((M, K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    dx = pk.linear_grad(dy.cuda(), x, w, need=(True, False, False))[0]
    assert torch.equal(dx.cpu(), e.sum(dim=1, keepdim=True).expand(M, K).bfloat16())
    # and along the rows
    dy = dy.t().contiguous().cuda()                                     # [N, M]
    x = torch.ones((N, K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    w = torch.zeros((M, K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    dw = pk.linear_grad(dy, x, w, need=(False, True, False))[1]
    assert torch.equal(dw.cpu(), e.sum(dim=1, keepdim=True).expand(M, K).bfloat16())


@pytest.mark.parametrize("M,K,N", [(3, 8, 5), (200, 72, 136)])
def test_infinite_and_largest_gradients(M, K, N):
    note(f"linear_grad of infinities {M}x{K}x{N}")
    inf = float("inf")
    dy = torch.zeros((M, N), device="cuda")
    dy[0, 1], dy[1, 2] = inf, -inf
    dy[2, 0] = torch.finfo(torch.float32).max                          # (past the largest bf16)
    w = torch.full((N, K), 0.5, dtype=torch.bfloat16, device="cuda")
    x = torch.full((M, K), 0.5, dtype=torch.bfloat16, device="cuda")
    dx, dw, _ = pk.linear_grad(dy, x, w)
    half = torch.tensor(2.0 ** 127)                                    # (half of it, to bf16)
    assert (dx[0] == inf).all() and (dx[1] == -inf).all() and (dx[2].float() == half).all() and (dx[3:] == 0).all()
    assert (dw[1] == inf).all() and (dw[2] == -inf).all() and (dw[0].float() == half).all() and (dw[3:] == 0).all()
    dy[0, 1] = float("nan")
    dx, dw, _ = pk.linear_grad(dy, x, w)
    assert torch.isnan(dx[0]).all() and torch.isnan(dw[1]).all()


@pytest.mark.parametrize("M,K,N", [(33, 64, 40), (200, 1001, 136)])
def test_rounded_by_choice(M, K, N):
    note(f"linear_grad rounded {M}x{K}x{N}")
    x, w, b, g = _inputs(M, K, N, 3)
    dy = torch.randn((M, N), generator=g).cuda()
    got = pk.linear_grad(dy, x, w, round_dz=True)
    want = pk.linear_grad(dy.bfloat16(), x, w)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(got[2], pk.linear_grad(dy, x, w)[2])            # (the bias's: from dz itself)
    assert not torch.equal(got[0], pk.linear_grad(dy, x, w)[0])
    # and through autograd
    for act, rounded in ((None, True), ("gelu", True), ("gelu", False)):
        leaves = [t.clone().requires_grad_() for t in (x, w, b)]
        pk.linear(*leaves, activation=act, round_dz=rounded).backward(dy)
        z = torch.empty((M, N), device="cuda")
        pk.linear(x, w, b, act, pre=z)
        for leaf, t in zip(leaves, pk.linear_grad(dy, x, w, z, act, round_dz=rounded)):
            assert torch.equal(leaf.grad, t)


def test_repeats():
    note("linear_grad in two terms, repeated")
    x, w, b, g = _inputs(600, 96, 80, 7)
    dy = torch.randn((600, 80), generator=g).cuda()
    full = pk.linear_grad(dy, x, w)
    for need in ((True, True, True), (True, False, False), (False, True, False), (False, False, True)):
        for p, f, k in zip(pk.linear_grad(dy, x, w, need=need), full, need):
            assert torch.equal(p, f) if k else p is None
