"""layer_norm, linear, adjust_logits and their gradients refuse what they cannot
take before anything is enqueued (host only: the dummy pointers are never
read)."""

import ctypes

import pytest
import torch

import paper_2608_12573_amd as pk


def _raises(fn, match):
    with pytest.raises(pk.ProfkError, match=match):
        fn()


def _at(n):
    return ctypes.c_void_p(n << 32)


A, B, C, D, E, F = (_at(n) for n in range(1, 7))
ODD1, ODD2 = ctypes.c_void_p((1 << 32) + 1), ctypes.c_void_p((1 << 32) + 2)


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=5), pk.EDTYPE), (dict(pdt=2), pk.EDTYPE), (dict(odt=-1), pk.EDTYPE), (dict(T=-1), pk.EINVAL),
    (dict(D=0), pk.EINVAL), (dict(D=2**20 + 1, st=2**21, ost=2**21), pk.EINVAL), (dict(st=99), pk.EINVAL),
    (dict(ost=99), pk.EINVAL), (dict(st=2**62), pk.EINVAL), (dict(eps=-1.0), pk.EINVAL), (dict(eps=0.0), pk.EINVAL),
    (dict(eps=float("nan")), pk.EINVAL), (dict(eps=float("inf")), pk.EINVAL), (dict(x=None), pk.ENULL),
    (dict(out=None), pk.ENULL), (dict(x=ODD2), pk.EINVAL), (dict(w=ODD1, pdt=1), pk.EINVAL), (dict(m=ODD2), pk.EINVAL),
    (dict(out=A, ost=101), pk.EINVAL), (dict(out=A, odt=1), pk.EINVAL),
    (dict(out=ctypes.c_void_p((1 << 32) + 4 * 299)), pk.EINVAL), (dict(T=0, x=None, out=None), pk.OK)])
def test_layer_norm_refusals(kw, rc):
    def call(dt=0, x=A, T=3, D=100, st=100, pdt=0, w=B, b=C, eps=1e-5, odt=0, out=D, ost=100, m=E, r=F):
        return pk.lib().profk_layer_norm(dt, x, T, D, st, pdt, w, b, eps, odt, out, ost, m, r, None)
    if "D" not in kw:
        kw = dict(kw, D=100)
    if "out" not in kw:
        kw = dict(kw, out=D)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=5), pk.EDTYPE), (dict(ddt=2), pk.EDTYPE), (dict(pdt=9), pk.EDTYPE), (dict(n=0), pk.EINVAL),
    (dict(T=2**31), pk.EINVAL), (dict(dst=99), pk.EINVAL), (dict(ost=99), pk.EINVAL), (dict(x=None), pk.ENULL),
    (dict(dy=None), pk.ENULL), (dict(m=None), pk.ENULL), (dict(r=None), pk.ENULL), (dict(ws=None), pk.ENULL),
    (dict(dx=A), pk.EINVAL), (dict(dx=B), pk.EINVAL), (dict(dy=ODD2), pk.EINVAL), (dict(dw=ODD2), pk.EINVAL),
    (dict(ws=ctypes.c_void_p((6 << 32) + 8)), pk.EINVAL), (dict(nb=64), pk.EWORKSPACE),
    (dict(T=0, dw=None, db=None), pk.OK), (dict(dx=None, dw=None, db=None), pk.OK)])
def test_layer_norm_grad_refusals(kw, rc):
    def call(dt=0, x=A, T=3, n=100, st=100, ddt=0, dy=B, dst=100, pdt=0, w=C, m=D, r=D, dx=E, ost=100, dw=D, db=D, ws=F,
             nb=1 << 20):
        return pk.lib().profk_layer_norm_grad(dt, x, T, n, st, ddt, dy, dst, pdt, w, m, r, dx, ost, dw, db, ws, nb, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(odt=4), pk.EDTYPE), (dict(K=0, xs=9, wst=9), pk.EINVAL), (dict(K=2**20 + 1, xs=2**21, wst=2**21), pk.EINVAL),
    (dict(M=-1), pk.EINVAL), (dict(N=2**31), pk.EINVAL), (dict(xs=99), pk.EINVAL), (dict(wst=99), pk.EINVAL),
    (dict(act=4), pk.EINVAL), (dict(act=-1), pk.EINVAL), (dict(rs=49), pk.EINVAL), (dict(x=None), pk.ENULL),
    (dict(w=None), pk.ENULL), (dict(out=None), pk.ENULL), (dict(x=ODD1), pk.EINVAL), (dict(b=ODD2), pk.EINVAL),
    (dict(out=A), pk.EINVAL), (dict(out=B), pk.EINVAL), (dict(pre=E), pk.EINVAL), (dict(pre=D), pk.EINVAL),
    (dict(out=D, rs=51), pk.EINVAL), (dict(out=C), pk.EINVAL), (dict(M=0, x=None), pk.OK),
    (dict(N=0, wst=100, out=None), pk.OK)])
def test_linear_refusals(kw, rc):
    def call(x=A, M=3, K=100, xs=100, w=B, N=50, wst=100, b=C, act=2, odt=0, r=D, rs=50, out=E, pre=F, ws=None, nb=0):
        n = pk.lib().profk_linear_workspace_size(M, K, N)
        return pk.lib().profk_linear(x, M, K, xs, w, N, wst, b, act, odt, r, rs, out, pre, _at(9) if n else ws, n or nb, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=4), pk.EDTYPE), (dict(K=0, xs=9, wst=9), pk.EINVAL), (dict(dst=49), pk.EINVAL), (dict(act=7), pk.EINVAL),
    (dict(dy=None), pk.ENULL), (dict(pre=None), pk.ENULL), (dict(x=None), pk.ENULL), (dict(w=None), pk.ENULL),
    (dict(ws=None), pk.ENULL), (dict(dx=A), pk.EINVAL), (dict(dw=B), pk.EINVAL), (dict(dw=E), pk.EINVAL),
    (dict(dx=C), pk.EINVAL), (dict(nb=16), pk.EWORKSPACE), (dict(ws=ctypes.c_void_p((9 << 32) + 8)), pk.EINVAL),
    (dict(dx=None, dw=None, db=None), pk.OK), (dict(M=0, dw=None, db=None), pk.OK)])
def test_linear_grad_refusals(kw, rc):
    def call(dt=0, dy=C, dst=50, pre=D, act=2, x=A, M=3, K=100, xs=100, w=B, N=50, wst=100, dx=E, dw=F, db=_at(8),
             ws=_at(9), nb=1 << 30):
        return pk.lib().profk_linear_grad(dt, dy, dst, pre, act, x, M, K, xs, w, N, wst, dx, dw, db, ws, nb, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=2), pk.EDTYPE), (dict(V=0), pk.EINVAL), (dict(V=2**31, st=2**31, ost=2**31), pk.EINVAL),
    (dict(st=99), pk.EINVAL), (dict(ost=99), pk.EINVAL), (dict(nt=-1), pk.EINVAL), (dict(nt=2**30), pk.EINVAL),
    (dict(nb=-1), pk.EINVAL), (dict(nb=2**30), pk.EINVAL), (dict(nm=0), pk.EINVAL), (dict(ast=3), pk.EINVAL), (dict(mask=None, nm=2), pk.EINVAL),
    (dict(x=None), pk.ENULL), (dict(off=None), pk.ENULL), (dict(out=None), pk.ENULL), (dict(bv=None), pk.ENULL),
    (dict(bo=None), pk.ENULL), (dict(tok=ctypes.c_void_p((2 << 32) + 4)), pk.EINVAL), (dict(al=ODD2), pk.EINVAL),
    (dict(x=ODD2), pk.EINVAL), (dict(out=A, ost=101), pk.EINVAL),
    (dict(out=ctypes.c_void_p((1 << 32) + 4)), pk.EINVAL), (dict(T=0, x=None), pk.OK)])
def test_adjust_refusals(kw, rc):
    def call(dt=0, x=A, T=3, V=100, st=100, tok=B, off=B, nt=5, np_=B, rep=B, pres=B, freq=B, bi=C, bv=C, bo=C, nb=4, al=D,
             nm=2, ast=4, mask=D, out=E, ost=100):
        return pk.lib().profk_adjust_logits(dt, x, T, V, st, tok, off, nt, np_, rep, pres, freq, bi, bv, bo, nb, al, nm,
                                            ast, mask, out, ost, None)
    assert call(**kw) == rc


@pytest.mark.parametrize("kw,rc", [
    (dict(dt=2), pk.EDTYPE), (dict(dst=99), pk.EINVAL), (dict(d=None), pk.ENULL), (dict(x=None), pk.ENULL),
    (dict(out=A), pk.EINVAL), (dict(out=F, ost=101), pk.EINVAL), (dict(nm=5, mask=None), pk.EINVAL),
    (dict(T=0, d=None), pk.OK)])
def test_adjust_grad_refusals(kw, rc):
    def call(dt=0, d=F, dst=100, x=A, T=3, V=100, st=100, tok=B, off=B, nt=5, rep=B, al=D, nm=2, ast=4, mask=D, out=E,
             ost=100):
        return pk.lib().profk_adjust_logits_grad(dt, d, dst, x, T, V, st, tok, off, nt, rep, al, nm, ast, mask, out, ost,
                                                 None)
    assert call(**kw) == rc


def test_sizes():
    L = pk.lib()
    assert L.profk_layer_norm_grad_workspace_size(0, 100) >= 800
    assert L.profk_layer_norm_grad_workspace_size(5, 0) == 0 == L.profk_layer_norm_grad_workspace_size(-1, 5)
    assert L.profk_linear_workspace_size(0, 8, 8) == 0 == L.profk_linear_workspace_size(8, 0, 8)
    assert L.profk_linear_grad_workspace_size(8, 0, 8) == 0
    for M, N in ((0, 8), (8, 0), (0, 0), (2**31 - 1, 2**31 - 1)):
        L.profk_linear_grad_workspace_size(M, 8, N)         # (whatever it is: sizes of nothing end no process)


def test_binding_refusals():
    x = torch.zeros(4, 64)
    b = x.bfloat16()
    _raises(lambda: pk.layer_norm(x), "CUDA tensor")
    _raises(lambda: pk.layer_norm(x.half()), "unsupported dtype")
    _raises(lambda: pk.layer_norm(x.t()), "unit column stride")
    _raises(lambda: pk.layer_norm_grad(x, x, None, x[:, 0], x[:, 0]), "CUDA tensor")
    _raises(lambda: pk.linear(b, b), "CUDA tensor")
    _raises(lambda: pk.linear_grad(x, b, b), "CUDA tensor")
    _raises(lambda: pk._activation("tanh"), "activation")
    _raises(lambda: pk.adjust_logits(x), "CUDA tensor")
    _raises(lambda: pk.adjust_logits_grad(x, x), "CUDA tensor")
    _raises(lambda: pk._history(4, 64, torch.zeros(3), None, None, None, None, None), "together")
    _raises(lambda: pk._history(4, 64, None, None, None, None, torch.zeros(4), None), "not given")
    _raises(lambda: pk._history(4, 64, None, None, None, torch.zeros(2, 3, dtype=torch.int32), None, None), "masks, 2")
    _raises(lambda: pk._params(torch.zeros(5), None, 6, None), "shape")
    _raises(lambda: pk._params(torch.zeros(6).half(), None, 6, None), "unsupported dtype")
    # no GPU is current here: tensors of another one are refused
    if not torch.cuda.is_available():
        return
    _raises(lambda: pk._stream_on(torch.device("cuda", 7)), "not the current device")
