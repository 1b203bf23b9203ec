"""Sums over the rows of matrices of more than 2^32 elements: the weights' and shifts'
gradients of linear and layer_norm against sums in 64 bits.

Tolerances, u = 2^-24: a product over M rows is within (M + 2) u of its terms'
magnitudes (twice that where dz comes as two terms, and 2^-16 of them for dz itself),
and half a step of bf16.  The norm's sums are taken by as many workgroups as the GPU
has CUs or more, 64 at least, each over its rows one after the other, and joined in
fewer than 64 additions: (T / 64 + 64) u of the terms' magnitudes, each term within 4 u
of itself and, by x - m, 2 u of (|x| + |m|) r |dy|; fp32 results."""

import pytest
import torch

import paper_2608_12573_amd as pk
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
BF = torch.finfo(torch.bfloat16).eps / 2


@pytest.fixture(autouse=True)
def _room():
    yield
    torch.cuda.empty_cache()


def _matrix(R, C, seed, dtype):
    """R rows, of which those of each 1000 are of their own size."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((R, C), dtype=dtype, device="cuda")
    base = torch.randn((1000, C), generator=g, device="cuda")
    for r in range(0, R, 1000):
        n = min(1000, R - r)
        x[r:r + n] = base[:n] * (0.5 + r / R)
    return x


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_product_over_the_rows(dtype):
    M, K, N = 66_001, 8, 66_000
    note(f"linear_grad's dW over {M}x{N} {dtype}")
    dy = _matrix(M, N, 1, dtype)
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((M, K), generator=g, device="cuda").bfloat16()
    w = torch.randn((N, K), generator=g, device="cuda").bfloat16()
    _, dw, db = pk.linear_grad(dy, x, w, need=(False, True, True))
    want, size = (torch.zeros((K, N), dtype=torch.float64, device="cuda") for _ in range(2))
    sums, mags = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2))
    for r in range(0, M, 2000):
        d, xt = dy[r:r + 2000].double(), x[r:r + 2000].double().t().contiguous()
        want += torch.mm(xt, d)
        size += torch.mm(xt.abs(), d.abs())
        sums += d.sum(dim=0)
        mags += d.abs().sum(dim=0)
    two = dtype is torch.float32
    tol = ((2 * M + 3) * U * 1.01 + 2.0 ** -16 if two else (M + 2) * U) * size + BF * want.abs()
    assert ((dw.double().t() - want).abs() <= tol).all()
    assert ((db.double() - sums).abs() <= (M + 20) * U * mags).all()
    # (the last rows count: without them the sums are others)
    short, _ = pk.linear_grad(dy[:-500], x[:-500], w, need=(False, True, False))[1:]
    assert not torch.equal(short, dw)


def test_norm_over_the_rows():
    T, D = 530_000, 8192
    note(f"layer_norm_grad's sums over {T}x{D}")
    x, dy = _matrix(T, D, 3, torch.bfloat16), _matrix(T, D, 4, torch.bfloat16)
    weight = torch.ones(D, device="cuda")
    m, r = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    for a in range(0, T, 10_000):
        _, m[a:a + 10_000], r[a:a + 10_000] = pk.layer_norm(x[a:a + 10_000], weight)
    _, dw, db = pk.layer_norm_grad(dy, x, weight, m, r, need=(False, True, True))
    want, size, sums, mags = (torch.zeros(D, dtype=torch.float64, device="cuda") for _ in range(4))
    for a in range(0, T, 10_000):
        d, mean, scale = dy[a:a + 10_000].double(), m[a:a + 10_000, None].double(), r[a:a + 10_000, None].double()
        v = x[a:a + 10_000].double()
        n = (v - mean) * scale
        want += (d * n).sum(dim=0)
        size += (d * n).abs().sum(dim=0) * (T / 64 + 68) + (2 * (v.abs() + mean.abs()) * scale * d.abs()).sum(dim=0)
        sums += d.sum(dim=0)
        mags += d.abs().sum(dim=0)
    assert ((dw.double() - want).abs() <= U * (size + want.abs())).all()
    assert ((db.double() - sums).abs() <= U * ((T / 64 + 64) * mags + sums.abs())).all()
