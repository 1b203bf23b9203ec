"""O5: microscaled 4-bit floating point, in fp64.

Test infrastructure (see the package docstring).  The format is MXFP4 of the
OCP Microscaling Formats specification 1.0: blocks of 32 values along a row,
one scale 2^s per block held as the byte s + 127 (255: NaN), values E2M1.
"""

import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])   # by code; 8 more with the sign


def padded(K):
    return -(-K // 128) * 128


def quantize(x):
    """(codes 0..15 [R, Kp], scale bytes [R, Kp / 32]) of fp32-valued x."""
    x = np.asarray(x, dtype=np.float64)
    R, K = x.shape
    v = np.zeros((R, padded(K)))
    v[:, :K] = x
    v = v.reshape(R, -1, 32)
    a = np.abs(v)
    bad = ~np.isfinite(v).all(axis=2)
    m = np.where(bad, 1.0, np.where(np.isfinite(a), a, 0.0).max(axis=2))
    # floor(log2 m), exactly: m = f 2^e with f in [0.5, 1)
    s = np.clip(np.where(m > 0, np.frexp(m)[1] - 1 - 2, -127), -127, 127)
    y = np.where(bad[:, :, None], 0.0, a) / np.ldexp(1.0, s)[:, :, None]
    mids = (GRID[1:] + GRID[:-1]) / 2
    # codes passed: a tie goes to the even one of its two neighbours
    code = sum(((y > mid) | ((y == mid) & (i % 2 == 1))).astype(np.int64) for i, mid in enumerate(mids))
    code |= np.where(np.signbit(v) & ~bad[:, :, None], 8, 0)
    byte = np.where(bad, 255, s + 127)
    return code.reshape(R, -1), byte


def pack(code):
    """Codes as bytes, the even value of a pair in the low half."""
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8)


def values(code, byte, K):
    """The values that codes and scale bytes stand for, [R, K]."""
    R = code.shape[0]
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    scale = np.where(byte == 255, np.nan, np.ldexp(1.0, np.minimum(byte, 254).astype(np.int64) - 127))
    return (v.reshape(R, -1, 32) * scale[:, :, None]).reshape(R, -1)[:, :K]


def round_trip(x):
    code, byte = quantize(x)
    return values(code, byte, np.asarray(x).shape[1])
