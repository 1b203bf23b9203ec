"""Every output of masked, unusual and ordered rows where a workgroup takes a
row in several steps: the kernel of long prompts (more rows than are split).

Tolerances, with u = 2^-24: a lane sums at most V/256 + 64 terms, each off by a
few u, and the row's last step is 64-bit and rounds once; the entropy's terms are
at most H + 2 in size, no exponent of its sums being above 1/2."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from oracle import logprobs as olp
from gpu_util import note, torch
from test_gpu_logprobs import KINDS, U24, _device_rows, _masked, _same, _size

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,n", [(9000, 20), (70001, 5), (9000, 0)])
def test_all_outputs_of_unsplit_rows(V, n, dtype, kind):
    t = torch()
    T = 1027
    x = _masked(kind, 6, V, 11)
    g, v = _device_rows(x, dtype)
    g = g.repeat(-(-T // 6), 1)[:T]
    y = (np.arange(T, dtype=np.int64) % 6) * (V // 7) - (np.arange(T) % 6 == 5)
    note(f"{kind} {dtype} T={T} V={V} n={n}")
    lp, h, lse, top, idx = [o[:6].cpu().numpy() for o in pk.token_logprobs(g, t.from_numpy(y).cuda(), n)]
    rlp, rh, rlse, rtop, ridx = olp.rows(v, y[:6], n)
    terms = V / 256 + 64
    assert np.array_equal(idx, ridx)
    _same(lse, rlse, U24 * (terms + 2 * _size(rlse)))
    _same(lp, rlp, U24 * (terms + 2 * _size(rlp)))
    _same(top, rtop, U24 * (terms + 2 * _size(rtop)))
    _same(h, rh, U24 * terms * (_size(rh) + 2))
    assert not (h < 0).any()
