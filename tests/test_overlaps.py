"""Outputs of layer_norm, linear, adjust_logits and their gradients that lie over an
input or another output are refused before anything is enqueued (host only: the
dummy pointers are never read)."""

import ctypes

import pytest

import paper_2608_12573_amd as pk

BASE = 1 << 32


def _at(i, off=0):
    return ctypes.c_void_p((i + 1) * BASE + off)


def _refused(call, names, outs, ins, n=24):
    """Each output over the first bytes of every input and of every other output,
    and over their last of n."""
    place = {k: _at(i) for i, k in enumerate(names)}
    for o in outs:
        for other in list(ins) + [p for p in outs if p != o]:
            for off in (0, n - 8, 8 - n):
                at = ctypes.c_void_p(place[other].value + off)
                assert call(**dict(place, **{o: at})) == pk.EINVAL, (o, other, off)


# (rows of 3 and 8 numbers: fp32 vectors of 24 bytes, or more)
@pytest.mark.parametrize("dt", [0, 1])
def test_layer_norm(dt):
    def call(x, w, b, out, m, r):
        return pk.lib().profk_layer_norm(dt, x, 6, 12, 12, 0, w, b, 1e-5, dt, out, 12, m, r, None)
    names = ("x", "w", "b", "out", "m", "r")
    _refused(call, names, ("out", "m", "r"), ("w", "b"))
    _refused(call, names, ("m", "r"), ("x", "w", "b"))
    place = {k: _at(i) for i, k in enumerate(names)}
    assert call(**dict(place, out=_at(0, 8))) == pk.EINVAL


@pytest.mark.parametrize("dt", [0, 1])
def test_layer_norm_grad(dt):
    need = pk.lib().profk_layer_norm_grad_workspace_size(6, 12)

    def call(x, dy, w, m, r, dx, dw, db, ws):
        ws = ctypes.c_void_p(ws.value // 16 * 16)
        return pk.lib().profk_layer_norm_grad(dt, x, 6, 12, 12, dt, dy, 12, 0, w, m, r, dx, 12, dw, db, ws, need, None)
    _refused(call, ("x", "dy", "w", "m", "r", "dx", "dw", "db", "ws"), ("dx", "dw", "db", "ws"), ("x", "dy", "w", "m", "r"))


@pytest.mark.parametrize("M", [6, 40])
def test_linear(M):
    need = pk.lib().profk_linear_workspace_size(M, 12, 12)
    assert need

    def call(x, w, b, r, out, pre, ws):
        ws = ctypes.c_void_p(ws.value // 16 * 16)
        return pk.lib().profk_linear(x, M, 12, 12, w, 12, 12, b, 1, 0, r, 12, out, pre, ws, need, None)
    names = ("x", "w", "b", "r", "out", "pre", "ws")
    _refused(call, names, ("out", "pre", "ws"), ("x", "w", "b"))
    _refused(call, names, ("pre", "ws"), ("r",))


def test_linear_grad():
    need = pk.lib().profk_linear_grad_workspace_size(6, 12, 12)

    def call(dy, pre, x, w, dx, dw, db, ws):
        ws = ctypes.c_void_p(ws.value // 16 * 16)
        return pk.lib().profk_linear_grad(0, dy, 12, pre, 2, x, 6, 12, 12, w, 12, 12, dx, dw, db, ws, need, None)
    _refused(call, ("dy", "pre", "x", "w", "dx", "dw", "db", "ws"), ("dx", "dw", "db", "ws"), ("dy", "pre", "x", "w"))


def test_adjust_logits():
    def call(x, tok, off, np_, rep, pres, freq, bi, bv, bo, al, mask, out):
        return pk.lib().profk_adjust_logits(0, x, 6, 100, 100, tok, off, 6, np_, rep, pres, freq, bi, bv, bo, 6, al, 2, 4,
                                            mask, out, 100, None)
    names = ("x", "tok", "off", "np_", "rep", "pres", "freq", "bi", "bv", "bo", "al", "mask", "out")
    _refused(call, names, ("out",), names[1:-1])

    def grad(d, x, tok, off, rep, al, mask, out):
        return pk.lib().profk_adjust_logits_grad(0, d, 100, x, 6, 100, 100, tok, off, 6, rep, al, 2, 4, mask, out, 100, None)
    names = ("d", "x", "tok", "off", "rep", "al", "mask", "out")
    _refused(grad, names, ("out",), names[1:-1])
