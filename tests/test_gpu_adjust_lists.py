"""adjust_logits with rows of many biases, whose cost is a pass over the list, not
one for each biased token; tolerances as in test_gpu_adjust."""

import pytest
import torch

import paper_2608_12573_amd as pk
from tests.gpu_util import note
from tests.test_gpu_adjust import _case, _check, _want

pytestmark = pytest.mark.gpu


def _dense(T, V, dtype, seed, per_token, history=40):
    """Every token biased per_token times, in an order of its own; the last row's
    list is empty."""
    x, kw = _case(T, V, dtype, seed, history=history, biases=0)
    g = torch.Generator().manual_seed(seed + 1)
    n = per_token * V
    ids = torch.cat([torch.randperm(n, generator=g) % V for _ in range(T - 1)])
    at = torch.arange(T + 1) * n
    at[T] = at[T - 1]
    kw["bias"] = (ids.cuda(), (4 * torch.randn(len(ids), generator=g)).cuda(), at.cuda())
    return x, kw


@pytest.mark.parametrize("V", [300, 2049, 16384, 16385, 40001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,per_token", [(3, 2), (40, 1)])
def test_every_token_biased(V, dtype, T, per_token):
    note(f"adjust_logits {per_token} biases for each of {T}x{V} {dtype}")
    x, kw = _dense(T, V, dtype, V, per_token)
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [8, 15, 16, 17, 31, 32, 33, 63, 64, 65, 255, 256, 257, 1000])
@pytest.mark.parametrize("V", [20000, 300])
def test_biases_about_the_listed_number(dtype, n, V):
    """n biases on neighbouring tokens of one piece, the row's others elsewhere."""
    note(f"adjust_logits {n} biases of {V} {dtype}")
    x, kw = _case(40, V, dtype, n, history=200, biases=0)
    g = torch.Generator().manual_seed(n)
    ids = torch.cat([torch.arange(n), torch.randint(-1, V + 1, (40,), generator=g)])
    ids = torch.cat([ids[torch.randperm(len(ids), generator=g)] % (V + 1) for _ in range(40)])
    kw["bias"] = (ids.cuda(), torch.randn(len(ids), generator=g).cuda(), (torch.arange(41) * (n + 40)).cuda())
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_histories_and_many_biases(dtype):
    note(f"adjust_logits long histories and many biases {dtype}")
    x, kw = _dense(4, 20001, dtype, 7, 1, history=40000)
    _check(pk.adjust_logits(x, **kw), *_want(x, kw), dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_alone(dtype):
    note(f"adjust_logits many biases in place {dtype}")
    x, kw = _dense(3, 9001, dtype, 8, 1)
    want = pk.adjust_logits(x, **kw)
    out = x.clone()
    assert pk.adjust_logits(out, out=out, **kw) is out and torch.equal(out, want)
    only = dict(bias=kw["bias"])
    _check(pk.adjust_logits(x, **only), *_want(x, only), dtype)


def test_longest_list():
    """400000 biases of one row, those of each token in ascending order: the last of
    each is its value."""
    note("adjust_logits 400000 biases of a row")
    V, n = 131072, 400000
    ids = torch.arange(n, device="cuda") % V
    values = torch.arange(n, device="cuda", dtype=torch.float32)
    at = torch.tensor([0, n], device="cuda")
    for dt in (torch.float32, torch.bfloat16):
        y = pk.adjust_logits(torch.zeros((1, V), dtype=dt, device="cuda"), bias=(ids, values, at))
        last = torch.arange(V, device="cuda") + (n - 1 - torch.arange(V, device="cuda")) // V * V
        assert torch.equal(y[0], last.float().to(dt))
    # all of them on one token
    y = pk.adjust_logits(torch.zeros((1, V), device="cuda"), bias=(ids * 0 + 77, values, at))
    assert y[0, 77] == n - 1 and int((y != 0).sum()) == 1

