"""The 4-bit product where a workgroup takes several groups of columns or
several tiles: more of them than the grid has workgroups (256 CUs).

Tolerance as for the other sizes: terms are exact, and the sum of the terms'
magnitudes s bounds an fp32 result's error by (K / 64 + 2) 2^-23 s."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from gpu_util import note, torch
from test_gpu_mx4 import _pair

pytestmark = pytest.mark.gpu

# few rows whose waves share the steps, a small and a larger a; tiles of 128 x
# 128, parts of stages and whole ones
SIZES = [(1, 20001, 1024), (2, 30000, 1000), (4, 8193, 4096), (20, 12001, 2048), (9, 30001, 1500), (100, 70001, 300),
         (200, 50001, 512)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_more_columns_than_workgroups(M, N, K):
    t = torch()
    note(f"mx4 product, several groups or tiles a workgroup: M={M} N={N} K={K}")
    x, qa, qb, ref, scale = _pair(M, N, K, M + N + K)
    tol = (K / 64 + 2) * 2.0 ** -23 * scale
    f = pk.mx4_matmul(*qa, *qb, K)
    err = np.abs(f.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err - tol).max()
    assert t.equal(pk.mx4_matmul(*qa, *qb, K, t.bfloat16), f.bfloat16())
    assert t.equal(pk.mx4_linear(x, *qb), f)
