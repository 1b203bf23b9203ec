"""The activations of linear and their slopes, at given z, in relative terms: small
results of the negative tail are as near as large ones.

z is the bias (of a product of zeros).  Phi, the sigmoid and e^(-z^2 / 2) are computed
to 2^-20 of themselves; gelu and silu round a product more, their slopes a few sums of
terms of the sizes s: 2^-19 of a result, or of s, and half a step of the output.
Below z = -12.5 (gelu) and -87 (silu) the results are 0 to 2e-36."""

import numpy as np
import pytest
import torch
from scipy.special import expit, log_ndtr

import paper_2608_12573_amd as pk
from tests.gpu_util import note

pytestmark = pytest.mark.gpu
REL = 2.0 ** -19


def _z(act):
    """From the least results to the largest, and the borders."""
    low = 12.5 if act == "gelu" else 87.0
    g = np.random.default_rng(1)
    z = np.concatenate([g.uniform(-low, low, 1500), -np.exp(g.uniform(np.log(1e-6), np.log(low), 1000)),
                        np.linspace(-1.0, 1.0, 501), [-low, 0.0, 1e-30, -1e-30, 13.0, 40.0, 41.0, 1e10]])
    return z.astype(np.float32)


def _value(z, act):
    return z * np.exp(log_ndtr(z)) if act == "gelu" else z * expit(z)


def _slope(z, act):
    """(the slope, the size of its terms)"""
    if act == "gelu":
        cdf, part = np.exp(log_ndtr(z)), z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
        return cdf + part, cdf + np.abs(part)
    p, q = expit(z), expit(-z)
    return p + z * p * q, p + np.abs(z) * p * q


# (few rows along k and across lanes, tiles, K in parts, operands at odd places)
@pytest.mark.parametrize("M,K,off", [(1, 64, 0), (3, 65, 0), (70, 64, 0), (300, 64, 0), (64, 4096, 0), (40, 64, 1)])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_values(M, K, off, act, dtype):
    note(f"{act} of {M}x{K} {dtype}, {off} in")
    z = _z(act)
    x = torch.zeros((M, K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    w = torch.zeros((len(z), K + off), dtype=torch.bfloat16, device="cuda")[:, off:]
    y = pk.linear(x, w, torch.from_numpy(z).cuda(), act, dtype=dtype).double().cpu().numpy()
    want = _value(z.astype(np.float64), act)
    assert (np.abs(y - want) <= (REL + torch.finfo(dtype).eps / 2) * np.abs(want) + 1e-38).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_slopes(act):
    note(f"slope of {act}")
    z = _z(act)
    one = torch.ones((1, len(z)), device="cuda")
    x, w = torch.zeros((1, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((len(z), 8), dtype=torch.bfloat16, device="cuda")
    got = pk.linear_grad(one, x, w, torch.from_numpy(z).cuda()[None], act, need=(False, False, True))[2].double().cpu().numpy()
    want, size = _slope(z.astype(np.float64), act)
    assert (np.abs(got - want) <= REL * size + 1e-36).all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_below_the_least(act):
    note(f"{act} below the least results")
    z = np.float32([-12.6, -13, -13.5, -14, -20, -39.9, -41, -87.1, -88, -90, -104, -200, -1e4, -3e38, -np.inf])
    x, w = torch.zeros((1, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((len(z), 8), dtype=torch.bfloat16, device="cuda")
    y = pk.linear(x, w, torch.from_numpy(z).cuda(), act).double().cpu().numpy()[0]
    with np.errstate(invalid="ignore"):
        want = np.where(np.isinf(z), 0.0, _value(z.astype(np.float64), act))
    assert (np.abs(y - want) <= REL * np.abs(want) + 2e-36).all()
    top = torch.tensor([float("inf"), 3e38], device="cuda")
    assert torch.equal(pk.linear(x, w[:2], top, act)[0], top)
