"""The 4-bit oracle: the nearest representable value by search, the block
scale's range, and its cases."""

import numpy as np
import pytest

from oracle import mx4 as omx


def test_nearest_value_by_search():
    g = np.random.default_rng(0)
    x = (g.standard_normal((4, 96)) * np.exp(g.standard_normal((4, 1)) * 3)).astype(np.float32)
    code, byte = omx.quantize(x)
    q = omx.values(code, byte, 96)
    for r in range(4):
        for b in range(3):
            blk = x[r, 32 * b:32 * b + 32].astype(np.float64)
            m = np.abs(blk).max()
            s = 2.0 ** (int(byte[r, b]) - 127)
            assert 4 * s <= m < 8 * s
            all_values = np.concatenate([omx.GRID, -omx.GRID]) * s
            for v, w in zip(blk, q[r, 32 * b:32 * b + 32]):
                assert abs(v - w) == np.abs(v - all_values).min()


@pytest.mark.parametrize("y,q", [(0.25, 0.0), (0.75, 1.0), (1.25, 1.0), (1.75, 2.0), (2.5, 2.0), (3.5, 4.0), (5.0, 4.0),
                                 (0.26, 0.5), (5.01, 6.0), (7.9, 6.0), (-2.5, -2.0), (-5.5, -6.0)])
def test_ties_to_even_and_saturation(y, q):
    x = np.zeros((1, 32), dtype=np.float32)
    x[0, 0], x[0, 1] = 4.0 if abs(y) < 4 else y, y   # the block's scale is 1
    assert omx.round_trip(x)[0, 1] == q


def test_special_blocks():
    x = np.zeros((1, 128), dtype=np.float32)
    x[0, 32] = np.inf
    x[0, 70] = np.nan
    x[0, 96] = 2.0 ** -149
    x[0, 97] = 2.0 ** -126
    code, byte = omx.quantize(x)
    assert byte[0].tolist() == [0, 255, 255, 0]
    q = omx.values(code, byte, 128)
    assert (q[0, :32] == 0).all() and np.isnan(q[0, 32:96]).all()
    assert q[0, 96] == 0 and q[0, 97] == 2.0 ** -126
    big = np.full((1, 32), np.finfo(np.float32).max, dtype=np.float32)
    assert omx.quantize(big)[1][0, 0] == 252 and omx.round_trip(big)[0, 0] == 6 * 2.0 ** 125


def test_idempotent_and_packed():
    g = np.random.default_rng(1)
    x = g.standard_normal((3, 77)).astype(np.float32)
    q = omx.round_trip(x)
    assert np.array_equal(omx.round_trip(q.astype(np.float32)), q)
    code, byte = omx.quantize(x)
    assert code.shape == (3, 128) and byte.shape == (3, 4) and omx.pack(code).shape == (3, 64)
    assert (code[:, 77:] == 0).all()
    assert omx.pack(np.array([[1, 15]]))[0, 0] == 0xF1
