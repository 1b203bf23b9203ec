"""token_logprobs and token_logprobs_grad refuse what they cannot take
before anything is enqueued (host only: the dummy pointers are never read)."""

import ctypes

import pytest
import torch

import paper_2608_12573_amd as pk


def _raises(fn, match):
    with pytest.raises(pk.ProfkError, match=match):
        fn()


def test_binding_refusals():
    x, y = torch.zeros(4, 16), torch.zeros(4, dtype=torch.int64)
    f = torch.zeros(4)
    _raises(lambda: pk.token_logprobs(x, y), "CUDA tensor")
    _raises(lambda: pk.token_logprobs(x[0], y), "2 dimension")
    _raises(lambda: pk.token_logprobs(x.half(), y), "unsupported dtype")
    _raises(lambda: pk.token_logprobs(x.t(), y), "unit column stride")
    _raises(lambda: pk.token_logprobs_grad(x, y, f, f, f), "CUDA tensor")
    _raises(lambda: pk.token_logprobs_grad(x.double(), y, f, f, f), "unsupported dtype")
    _raises(lambda: pk._vector(y.int(), "tokens", torch.int64, (4,), None), "tokens must be contiguous")
    _raises(lambda: pk._vector(f[:3], "lse", torch.float32, (4,), None), "shape")
    _raises(lambda: pk._vector(torch.zeros(8)[::2], "lse", torch.float32, (4,), None), "contiguous")
    _raises(lambda: pk._vector([0], "tokens", torch.int64, (1,), None), "torch tensor")


P = ctypes.c_void_p(4096)


def _fwd(dtype=0, x=P, T=8, V=100, stride=100, y=P, n=4, lp=P, h=P, lse=P, top=P, idx=P, ws=P, nb=1 << 30):
    return pk.lib().profk_token_logprobs(dtype, x, T, V, stride, y, n, lp, h, lse, top, idx, ws, nb, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dtype=2), pk.EDTYPE), (dict(T=-1), pk.EINVAL), (dict(T=2**31), pk.EINVAL), (dict(V=0, stride=1), pk.EINVAL),
    (dict(V=2**31, stride=2**31), pk.EINVAL), (dict(stride=99), pk.EINVAL), (dict(n=-1), pk.EINVAL),
    (dict(n=65), pk.EINVAL), (dict(stride=2**62), pk.EINVAL), (dict(x=None), pk.ENULL), (dict(y=None), pk.ENULL),
    (dict(lp=None), pk.ENULL), (dict(h=None), pk.ENULL), (dict(lse=None), pk.ENULL), (dict(top=None), pk.ENULL),
    (dict(idx=None), pk.ENULL), (dict(x=ctypes.c_void_p(4098)), pk.EINVAL),
    (dict(dtype=1, x=ctypes.c_void_p(4097)), pk.EINVAL), (dict(ws=ctypes.c_void_p(4104)), pk.EINVAL),
    (dict(V=131072, stride=131072, ws=None, nb=0), pk.ENULL), (dict(V=131072, stride=131072, nb=8), pk.EWORKSPACE)])
def test_forward_refusals(kw, rc):
    assert _fwd(**kw) == rc


def _bwd(dtype=0, x=P, T=8, V=100, stride=100, y=P, lse=P, h=P, gl=P, gh=P, n=4, idx=P, gt=P, out=ctypes.c_void_p(1 << 20), os=100):
    return pk.lib().profk_token_logprobs_grad(dtype, x, T, V, stride, y, lse, h, gl, gh, n, idx, gt, out, os, None)


@pytest.mark.parametrize("kw,rc", [
    (dict(dtype=-1), pk.EDTYPE), (dict(V=0), pk.EINVAL), (dict(os=99), pk.EINVAL), (dict(stride=1), pk.EINVAL),
    (dict(n=65), pk.EINVAL), (dict(x=None), pk.ENULL), (dict(lse=None), pk.ENULL), (dict(out=None), pk.ENULL),
    (dict(y=None), pk.ENULL), (dict(h=None), pk.ENULL), (dict(idx=None), pk.ENULL), (dict(gt=None), pk.ENULL),
    (dict(out=ctypes.c_void_p((1 << 20) + 2)), pk.EINVAL), (dict(os=2**62), pk.EINVAL), (dict(out=P), pk.EINVAL),
    (dict(out=ctypes.c_void_p(4096 + 400)), pk.EINVAL), (dict(x=ctypes.c_void_p((1 << 20) - 3196)), pk.EINVAL)])
def test_gradient_refusals(kw, rc):
    # (the last three: `out` overlaps the logits)
    assert _bwd(**kw) == rc


def test_no_rows_is_no_work():
    assert _fwd(T=0, x=None, y=None, lp=None) == pk.OK
    assert _bwd(T=0, x=None, lse=None, out=None) == pk.OK
    L = pk.lib()
    assert L.profk_token_logprobs_workspace_size(0, 100, 4) == 0
    assert L.profk_token_logprobs_workspace_size(4, 100, 65) == 0


def test_workspace_only_for_few_long_rows():
    size = pk.lib().profk_token_logprobs_workspace_size
    assert size(1, 131072, 20) > 0
    assert size(4096, 131072, 20) == 0
    assert size(1, 512, 8) == 0
    # statistics and alternatives of at most 256 chunks a row
    assert size(1, 2**31 - 1, 64) <= 256 * (16 + 64 * 8) + 256
