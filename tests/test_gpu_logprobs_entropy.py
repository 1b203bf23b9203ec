"""The entropy of confident rows: a few logits far above all others, so that
the sums have a few terms that matter and all others are 0 in fp32.

Tolerance, with u = 2^-24 and t the exponents of the kernels' sums: the largest
t lies within 1/2 of 0 and exp2 is off by 2 u of itself, which log2 s and q / s
both see (2.9 u and u), the logarithm by u, the products and the quotient by u
of 1/2 each; a second and a third term add two roundings to each sum (2.9 u and
u).  All of it times ln 2, and H's own rounding: under 8 u (1 + H)."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from gpu_util import note, torch

pytestmark = pytest.mark.gpu
TOL = 8 * 2.0 ** -24


def _entropies(x, dtype, n):
    """(the kernel's, the 64-bit) entropies of host rows x."""
    t = torch()
    g = t.from_numpy(x).cuda().to(t.float32 if dtype == "f32" else t.bfloat16)
    y = t.zeros(x.shape[0], dtype=t.int64, device="cuda")
    h = pk.token_logprobs(g, y, n)[1].double().cpu().numpy()
    v = g.double().cpu().numpy()
    with np.errstate(invalid="ignore", divide="ignore"):
        d = v - v.max(axis=1, keepdims=True)
        e = np.exp(d)
        s = e.sum(axis=1, keepdims=True)
        l = d - np.log(s)
        p = np.exp(l)
        ref = -np.where(p > 0, p * l, 0.0).sum(axis=1)
    return h, ref


# one wave; a workgroup's several steps; rows split over workgroups
SHAPES = [(1500, 700), (1500, 9000), (60, 131072)]


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("n", [0, 5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_logit_far_above(T, V, n, dtype):
    g = np.random.default_rng(V + n)
    for mask in (-np.inf, -300.0):
        x = np.full((T, V), mask, dtype=np.float32)
        x[np.arange(T), g.integers(0, V, T)] = g.uniform(-60.0, 60.0, T)
        note(f"entropy of one logit {dtype} T={T} V={V} n={n} mask={mask}")
        h, ref = _entropies(x, dtype, n)
        assert np.abs(ref).max() < 1e-60
        assert (h >= 0).all(), h.min()
        assert (h <= TOL).all(), h.max()


@pytest.mark.parametrize("T,V", SHAPES)
@pytest.mark.parametrize("n", [0, 5])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rising_logits_far_apart(T, V, n, dtype):
    """Two and three logits up to 16 powers of two apart, the larger ones later
    in the row."""
    g = np.random.default_rng(V + n + 1)
    x = np.full((T, V), -np.inf, dtype=np.float32)
    r = np.arange(T)
    top = g.uniform(-20.0, 20.0, T)
    x[r, g.integers(0, V // 16, T)] = top - g.uniform(8.0, 11.0, T)
    x[r, g.integers(V // 4, V // 2, T)] = top - g.uniform(5.0, 11.0, T)
    x[r, g.integers(V // 2, V, T)] = top
    note(f"entropy of rising logits {dtype} T={T} V={V} n={n}")
    h, ref = _entropies(x, dtype, n)
    err = np.abs(h - ref)
    assert (err <= TOL * (1 + ref)).all(), (err.max(), (err / (1 + ref)).max() / TOL)
