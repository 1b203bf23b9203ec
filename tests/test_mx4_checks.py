"""The 4-bit calls refuse what they cannot take before anything is enqueued
(host only: the dummy pointers are never read)."""

import ctypes

import pytest
import torch

import paper_2608_12573_amd as pk


def _raises(fn, match):
    with pytest.raises(pk.ProfkError, match=match):
        fn()


def test_sizes():
    L = pk.lib()
    assert L.profk_mx4_codes_size(3, 1) == 3 * 64 and L.profk_mx4_scales_size(3, 1) == 128
    assert L.profk_mx4_codes_size(5, 129) == 5 * 128 and L.profk_mx4_scales_size(33, 129) == 512
    assert L.profk_mx4_codes_size(2**31 - 1, 2**20) == (2**31 - 1) * 2**19
    for R, K in ((-1, 5), (5, 0), (5, 2**20 + 1), (2**31, 5)):
        assert L.profk_mx4_codes_size(R, K) == 0 and L.profk_mx4_scales_size(R, K) == 0
    assert L.profk_mx4_linear_workspace_size(33, 129, 7) == (33 * 128 + 255) // 256 * 256 + 512
    assert L.profk_mx4_linear_workspace_size(3, 129, 7) == 0      # few rows: none
    assert L.profk_mx4_linear_workspace_size(0, 129, 7) == 0


def test_binding_refusals():
    x = torch.zeros(4, 64)
    c, s = torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(1, 1, 32, 4, dtype=torch.uint8)
    _raises(lambda: pk.mx4_quantize(x), "CUDA tensor")
    _raises(lambda: pk.mx4_quantize(x.half()), "unsupported dtype")
    _raises(lambda: pk.mx4_quantize(x[0]), "2 dimension")
    _raises(lambda: pk.mx4_quantize(x.t()), "unit column stride")
    _raises(lambda: pk.mx4_dequantize(c, s, 64), "CUDA tensor")
    _raises(lambda: pk.mx4_dequantize(c, s, 129), "shape")
    _raises(lambda: pk.mx4_dequantize(c, s, 0), "from 1")
    _raises(lambda: pk.mx4_dequantize(c.int(), s, 64), "uint8")
    _raises(lambda: pk.mx4_matmul(c, s, c, s, 64), "CUDA tensor")
    _raises(lambda: pk.mx4_linear(x, c, s), "CUDA tensor")
    _raises(lambda: pk.mx4_outputs(3, 2**20 + 1, "cpu"), "from 1")


P = ctypes.c_void_p(4096)
ODD = ctypes.c_void_p(4098)


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=5), pk.EDTYPE), (dict(R=-1), pk.EINVAL), (dict(K=0), pk.EINVAL), (dict(K=2**20 + 1, st=2**21), pk.EINVAL),
    (dict(st=99), pk.EINVAL), (dict(st=2**62), pk.EINVAL), (dict(x=None), pk.ENULL), (dict(c=None), pk.ENULL),
    (dict(s=None), pk.ENULL), (dict(x=ODD), pk.EINVAL), (dict(c=ctypes.c_void_p(4104)), pk.EINVAL), (dict(s=ODD), pk.EINVAL),
    (dict(R=0, x=None), pk.OK)])
def test_quantize_refusals(kw, rc):
    def call(dt=0, x=P, R=3, K=100, st=100, c=P, s=P):
        return pk.lib().profk_mx4_quantize(dt, x, R, K, st, c, s, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=5), pk.EDTYPE), (dict(K=0), pk.EINVAL), (dict(c=None), pk.ENULL), (dict(o=None), pk.ENULL),
    (dict(o=ODD), pk.EINVAL), (dict(c=ODD), pk.EINVAL), (dict(R=0, o=None), pk.OK)])
def test_dequantize_refusals(kw, rc):
    def call(dt=0, c=P, s=P, R=3, K=100, o=P):
        return pk.lib().profk_mx4_dequantize(dt, c, s, R, K, o, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(od=7), pk.EDTYPE), (dict(M=-1), pk.EINVAL), (dict(N=2**31), pk.EINVAL), (dict(K=0), pk.EINVAL),
    (dict(a=None), pk.ENULL), (dict(bs=None), pk.ENULL), (dict(o=None), pk.ENULL), (dict(b=ODD), pk.EINVAL),
    (dict(as_=ODD), pk.EINVAL), (dict(o=ODD), pk.EINVAL), (dict(M=0, a=None), pk.OK), (dict(N=0, o=None), pk.OK)])
def test_matmul_refusals(kw, rc):
    def call(a=P, as_=P, M=4, b=P, bs=P, N=8, K=100, od=0, o=P):
        return pk.lib().profk_mx4_matmul(a, as_, M, b, bs, N, K, od, o, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=3), pk.EDTYPE), (dict(od=3), pk.EDTYPE), (dict(K=0), pk.EINVAL), (dict(st=99), pk.EINVAL),
    (dict(x=None), pk.ENULL), (dict(ws=None), pk.ENULL), (dict(nb=7), pk.EWORKSPACE), (dict(ws=ctypes.c_void_p(4104)), pk.EINVAL),
    (dict(w=ODD), pk.EINVAL), (dict(M=0, x=None), pk.OK), (dict(st=2**62), pk.EINVAL)])
def test_linear_refusals(kw, rc):
    def call(dt=0, x=P, M=40, K=100, st=100, w=P, s=P, N=8, od=0, o=P, ws=P, nb=1 << 20):
        return pk.lib().profk_mx4_linear(dt, x, M, K, st, w, s, N, od, o, ws, nb, None)
    assert call(**kw) == rc
