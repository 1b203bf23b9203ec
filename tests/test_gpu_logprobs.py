"""Token log probabilities, entropy, alternatives and their gradient on the
GPU against the fp64 oracle.

Tolerances, with u = 2^-24: a lane sums at most V/256 + 64 terms one after
another, each off by a few u, so that s is off by (V/256 + 64) u of itself at
worst; the row's last step is 64-bit and rounds once.  The entropy's sum has
terms of up to H + 32 in size.  A gradient's terms are off by a few u each,
p by u |x - lse| more (oracle.logprobs.grad_scale), and bf16 rounds the result
to 8 bits.  Alternatives are the same indices."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from oracle import logprobs as olp
from gpu_util import note, torch

pytestmark = pytest.mark.gpu
U24 = 2.0 ** -24


def _device_rows(x, dtype, pad=0, offset=0):
    """x (host fp32 [T, V]) on the GPU as `dtype`, rows `pad` elements further
    apart and the first `offset` elements into an allocation; and the fp64
    values that it holds."""
    t = torch()
    T, V = x.shape
    dt = t.float32 if dtype == "f32" else t.bfloat16
    big = t.full((offset + T * (V + pad),), float("nan"), dtype=dt, device="cuda")
    g = big[offset:].view(T, V + pad)[:, :V] if T else t.empty((0, V), dtype=dt, device="cuda")
    g.copy_(t.from_numpy(np.ascontiguousarray(x)).cuda().to(dt))
    return g, g.double().cpu().numpy()


def _same(got, ref, tol):
    got = np.asarray(got, dtype=np.float64)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    inf = ok & np.isinf(ref)
    assert np.array_equal(got[inf], ref[inf])
    fin = ok & ~inf
    assert np.isfinite(got[fin]).all()
    err = np.abs(got[fin] - ref[fin])
    tol = np.broadcast_to(tol, got.shape)[fin]
    assert (err <= tol).all(), (err.max(), tol[err.argmax()])


def _size(a):
    return np.where(np.isfinite(a), np.abs(a), 0.0)


def _check(x, y, n, dtype, pad=0, offset=0):
    t = torch()
    T, V = x.shape
    note(f"logprobs {dtype} T={T} V={V} n={n} pad={pad} offset={offset}")
    g, v = _device_rows(x, dtype, pad, offset)
    out = pk.token_logprobs(g, t.from_numpy(y).cuda(), n)
    t.cuda.synchronize()
    lp, h, lse, top, idx = [o.cpu().numpy() for o in out]
    rlp, rh, rlse, rtop, ridx = olp.rows(v, y, n)
    terms = V / 256 + 64
    _same(lse, rlse, U24 * (terms + 2 * _size(rlse)))
    _same(lp, rlp, U24 * (terms + 2 * _size(rlp)))
    _same(h, rh, U24 * terms * (_size(rh) + 32))
    assert np.array_equal(idx, ridx)
    _same(top, rtop, U24 * (terms + 2 * _size(rtop)))
    return g, v, out


def _x(T, V, seed, scale=3.0):
    return (np.random.default_rng(seed).standard_normal((T, V)) * scale).astype(np.float32)


def _tokens(T, V, seed):
    g = np.random.default_rng(seed + 100)
    return np.where(g.random(T) < 0.8, g.integers(0, V, T), -100).astype(np.int64)


SIZES = [(3, 1, 1), (2, 2, 5), (5, 3, 2), (4, 7, 7), (3, 63, 64), (7, 65, 20), (5, 512, 8), (3, 513, 64), (2, 1000, 0),
         (3, 2047, 20), (2, 2049, 1), (2, 4099, 33), (1, 16387, 20), (3, 50001, 20), (1, 131072, 20), (2, 131072, 64),
         (1, 262147, 5), (70, 9001, 20), (1030, 4111, 3), (1100, 100, 20), (1025, 10007, 64)]


@pytest.mark.parametrize("T,V,n", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_sizes(T, V, n, dtype):
    _check(_x(T, V, V + n), _tokens(T, V, V), n, dtype)


@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 3), (5, 7)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_offsets(pad, offset, dtype):
    _check(_x(5, 1003, 1), _tokens(5, 1003, 1), 20, dtype, pad, offset)
    _check(_x(1030, 777, 2), _tokens(1030, 777, 2), 20, dtype, pad, offset)
    _check(_x(2, 70001, 3), _tokens(2, 70001, 3), 20, dtype, pad, offset)


def _masked(kind, T, V, seed):
    x = _x(T, V, seed)
    g = np.random.default_rng(seed)
    low = np.float32(np.finfo(np.float32).min)
    if kind == "half":
        x[g.random((T, V)) < 0.5] = -np.inf
    elif kind == "few":          # fewer left than asked for
        keep = g.integers(0, V, (T, 5))
        m = np.ones((T, V), dtype=bool)
        np.put_along_axis(m, keep, False, axis=1)
        x[m] = -np.inf
    elif kind == "none":         # rows 0 and 2 allow nothing
        x[0] = -np.inf
        x[2] = -np.inf
    elif kind == "lowest":       # the lowest value as the mask, all or all but three
        x[:] = low
        x[1, [1, V // 2, V - 1]] = [0.5, 2.0, -1.0]
    elif kind == "range":        # all but a late range
        x[:, :V - V // 8] = -np.inf
    elif kind == "late":         # the first part lower, but not masked
        x[:, :V // 2] -= 1000.0
    elif kind == "nan":
        x[0, V // 3] = np.nan
        x[1, V - 1] = -np.float32(np.nan)
        x[2, 0] = np.inf
        x[2, 1] = -np.inf
    elif kind == "large":        # past the fast path's range, and far apart
        x[0] *= 1e37
        x[1] = 3e38
        x[2] *= 1e30
    elif kind == "low":          # at the lower end of the fast path's range
        x -= 1e6
        x[1] -= 90.0
        x[2] -= 3000.0
    elif kind == "rising":
        x.sort(axis=1)
    elif kind == "falling":
        x = -np.sort(-x, axis=1)
    elif kind == "equal":
        x[:] = 1.25
    elif kind == "steps":        # few different values, many ties
        x = np.round(x)
    elif kind == "zeros":
        x = np.where(g.random((T, V)) < 0.5, np.float32(0.0), np.float32(-0.0)).astype(np.float32)
    elif kind == "far":          # one value far above, thousands below
        x[:, 0] = 200.0
        x[:, 1:] -= 5000.0
    elif kind == "one_lane":     # the best all in places that one lane reads
        x[:, 8:16] += 100.0
        x[:, 0::2048] += 50.0
    return x


KINDS = ["half", "few", "none", "lowest", "range", "late", "nan", "large", "low", "rising", "falling", "equal", "steps", "zeros",
         "far", "one_lane"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_masks_and_orders(kind, dtype):
    for T, V, n in [(4, 333, 20), (3, 5000, 20), (3, 70001, 64), (1027, 9000, 20)]:
        x = _masked(kind, min(T, 6), V, 11)
        x = np.concatenate([x] * (-(-T // len(x))))[:T]
        if T > 1000:      # (the oracle takes the distinct rows; the rest repeat them)
            t = torch()
            g, v = _device_rows(x, dtype)
            y = np.arange(T, dtype=np.int64) % 6 * 7
            note(f"{kind} {dtype} T={T} V={V}")
            out = [o.cpu().numpy() for o in pk.token_logprobs(g, t.from_numpy(y).cuda(), n)]
            for o in out:
                for r in range(6, T):
                    assert np.array_equal(o[r], o[r % 6], equal_nan=True)
            assert np.array_equal(out[4][:6], olp.rows(v[:6], y[:6], n)[4])
        else:
            _check(x, _tokens(T, V, 5), n, dtype)


def test_tokens_outside():
    x = _x(4, 100, 3)
    _check(x, np.array([-1, 100, 99, 2**40], dtype=np.int64), 3, "f32")


def test_no_rows():
    t = torch()
    out = pk.token_logprobs(t.empty((0, 50), device="cuda"), t.empty(0, dtype=t.int64, device="cuda"), 4)
    assert [tuple(o.shape) for o in out] == [(0,), (0,), (0,), (0, 4), (0, 4)]
    d = pk.token_logprobs_grad(t.empty((0, 50), device="cuda"), t.empty(0, dtype=t.int64, device="cuda"),
                               out[0], out[1], out[2])
    assert tuple(d.shape) == (0, 50)


def test_rows_past_32_bit_offsets():
    """Rows that start past 2^32 elements into their allocation."""
    t = torch()
    T, V, stride = 3, 5001, (1 << 31) + 17
    big = t.empty(2 * stride + 2 * V, dtype=t.bfloat16, device="cuda")
    g = big.as_strided((T, V), (stride, 1))
    x = _x(T, V, 9)
    g.copy_(t.from_numpy(x).cuda().to(t.bfloat16))
    y = np.array([5, 4000, 17], dtype=np.int64)
    note("logprobs at 64-bit offsets")
    out = [o.cpu().numpy() for o in pk.token_logprobs(g, t.from_numpy(y).cuda(), 20)]
    ref = olp.rows(g.double().cpu().numpy(), y, 20)
    assert np.array_equal(out[4], ref[4])
    _same(out[0], ref[0], U24 * (100 + 2 * np.abs(ref[0])))
    one = t.ones(T, device="cuda")
    lse, h = (t.from_numpy(o).cuda() for o in (out[2], out[1]))
    yd = t.from_numpy(y).cuda()
    d = pk.token_logprobs_grad(g, yd, lse, h, one)
    e = pk.token_logprobs_grad(g.contiguous(), yd, lse, h, one)
    assert t.equal(d, e)
    o = big[V:].as_strided((T, V), (stride, 1))
    with pytest.raises(pk.ProfkError):      # between the logits' rows
        pk.token_logprobs_grad(g, yd, lse, h, one, out=o)
    assert t.equal(pk.token_logprobs_grad(g.contiguous(), yd, lse, h, one, out=o), e)


def _check_grad(x, y, dtype, n, pad=0, offset=0, entropy=True, token=True, seed=0):
    t = torch()
    T, V = x.shape
    note(f"grad {dtype} T={T} V={V} n={n} pad={pad} offset={offset}")
    g, v = _device_rows(x, dtype, pad, offset)
    yd = t.from_numpy(y).cuda()
    _, h, lse, _, idx = pk.token_logprobs(g, yd, n)
    r = np.random.default_rng(seed)
    gl = r.standard_normal(T).astype(np.float32) if token else None
    gh = r.standard_normal(T).astype(np.float32) if entropy else None
    gt = r.standard_normal((T, n)).astype(np.float32) if n else None
    idx = idx.clone()
    if n > 2:                    # an index twice, one outside, and the token
        idx[:, 1] = idx[:, 0]
        idx[::2, 2] = V + 3
        idx[1::2, 2] = yd[1::2]
    dev = lambda a: t.from_numpy(a).cuda() if a is not None else None
    out = t.full((T, V + pad), float("nan"), dtype=g.dtype, device="cuda")
    d = pk.token_logprobs_grad(g, yd, lse, h, dev(gl), dev(gh), idx if n else None, dev(gt), out=out[:, :V])
    assert t.isnan(out[:, V:]).all()
    t.cuda.synchronize()
    got = d.double().cpu().numpy()
    lse, h, idx = lse.double().cpu().numpy(), h.double().cpu().numpy(), idx.cpu().numpy()
    bf = dtype == "bf16"
    for k in range(T):
        a = (v[k], int(y[k]), lse[k], h[k], None if gl is None else float(gl[k]), None if gh is None else float(gh[k]),
             idx[k] if n else [], gt[k].astype(np.float64) if n else np.zeros(0))
        ref = olp.grad_row(*a)
        tol = U24 * olp.grad_scale(*a) + 1e-36 + (2.0 ** -8 * _size(ref) if bf else 0.0)
        _same(got[k], ref, tol)


@pytest.mark.parametrize("T,V,n", [(3, 1, 0), (3, 2, 1), (5, 3, 3), (4, 64, 0), (3, 65, 20), (9, 1000, 16), (2, 4099, 0),
                                   (3, 8192, 16), (2, 50001, 64), (1, 131072, 0), (200, 777, 3)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_sizes(T, V, n, dtype):
    _check_grad(_x(T, V, V), _tokens(T, V, V), dtype, n)


@pytest.mark.parametrize("entropy,token,n", [(False, True, 0), (True, False, 0), (False, False, 5), (True, True, 5)])
def test_gradient_parts(entropy, token, n):
    for dtype in ("f32", "bf16"):
        _check_grad(_x(6, 2051, 4), _tokens(6, 2051, 4), dtype, n, entropy=entropy, token=token, pad=5,
                    offset=3)


@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 3), (5, 7)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_strides(pad, offset, dtype):
    _check_grad(_x(5, 1003, 1), _tokens(5, 1003, 1), dtype, 16, pad, offset)
    _check_grad(_x(2, 9001, 1), _tokens(2, 9001, 1), dtype, 0, pad, offset)


@pytest.mark.parametrize("kind", ["half", "few", "none", "lowest", "nan", "large", "low", "equal", "far"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradient_masks(kind, dtype):
    _check_grad(_masked(kind, 5, 3001, 3), np.array([0, 5, 7, -1, 4000], dtype=np.int64), dtype, 8)


def test_gradient_equals_differences():
    """Against differences of the 64-bit forward pass, not of its formula."""
    t = torch()
    T, V, n = 3, 21, 4
    x, y = _x(T, V, 8, 1.5), np.array([0, 20, 7], dtype=np.int64)
    g, v = _device_rows(x, "f32")
    yd = t.from_numpy(y).cuda()
    note("grad against differences")
    _, h, lse, _, idx = pk.token_logprobs(g, yd, n)
    r = np.random.default_rng(2)
    gl, gh, gt = r.standard_normal(T), r.standard_normal(T), r.standard_normal((T, n))
    dev = lambda a: t.from_numpy(a.astype(np.float32)).cuda()
    d = pk.token_logprobs_grad(g, yd, lse, h, dev(gl), dev(gh), idx, dev(gt)).cpu().numpy()
    idx = idx.cpu().numpy()
    for k in range(T):
        def f(z):
            lp, hh, ls, _, _ = olp.row(z, int(y[k]), 0)
            return gl[k] * lp + gh[k] * hh + sum(gt[k, i] * (z[idx[k, i]] - ls) for i in range(n))
        e = 1e-5
        num = [(f(v[k] + e * np.eye(V)[j]) - f(v[k] - e * np.eye(V)[j])) / (2 * e) for j in range(V)]
        # the difference's own error is about 1e-9; the gradients are rounded to fp32 before
        assert np.abs(d[k] - num).max() < 2e-6


def test_other_stream_and_kept_buffers():
    """Calls on a side stream with a kept workspace and outputs, twice: the
    second call's results are its own."""
    t = torch()
    T, V, n = 2, 60001, 20
    a, va = _device_rows(_x(T, V, 1), "f32")
    b, vb = _device_rows(_x(T, V, 2), "f32")
    y = np.array([3, 59999], dtype=np.int64)
    yd = t.from_numpy(y).cuda()
    ws, out = pk.token_logprobs_workspace(T, V, n), pk.token_logprobs_outputs(T, n)
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    note("logprobs on a side stream")
    with t.cuda.stream(side):
        pk.token_logprobs(a, yd, n, ws=ws, out=out)
        first = [o.clone() for o in out]
        pk.token_logprobs(b, yd, n, ws=ws, out=out)
    side.synchronize()
    for o, v in ((first, va), (out, vb)):
        ref = olp.rows(v, y, n)
        assert np.array_equal(o[4].cpu().numpy(), ref[4])
        _same(o[0].cpu().numpy(), ref[0], U24 * (400 + 2 * np.abs(ref[0])))


def test_graph_replays():
    t = torch()
    T, V, n = 3, 40001, 20
    g, _ = _device_rows(_x(T, V, 1), "f32")
    yd = t.from_numpy(_tokens(T, V, 1)).cuda()
    ws, out = pk.token_logprobs_workspace(T, V, n), pk.token_logprobs_outputs(T, n)
    d = t.empty((T, V), device="cuda")
    one = t.ones(T, device="cuda")

    def call():
        pk.token_logprobs(g, yd, n, ws=ws, out=out)
        pk.token_logprobs_grad(g, yd, out[2], out[1], one, one, out[4], out[3], out=d)

    note("logprobs under capture")
    call()
    ref = [o.clone() for o in (*out, d)]
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        call()
    t.cuda.current_stream().wait_stream(side)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        call()
    for _ in range(3):
        for o in (*out, d):
            o.fill_(-7)
        ws.fill_(255)
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        for o, f in zip((*out, d), ref):
            assert t.equal(o, f)


def test_refusals_on_the_device():
    t = torch()
    x, y, f = t.zeros(4, 16, device="cuda"), t.zeros(4, dtype=t.int64, device="cuda"), t.zeros(4, device="cuda")
    bad = [lambda: pk.token_logprobs(x, y.int()), lambda: pk.token_logprobs(x, y[:3]),
           lambda: pk.token_logprobs(x, y.cpu()), lambda: pk.token_logprobs(x, y, 65), lambda: pk.token_logprobs(x, y, -1),
           lambda: pk.token_logprobs(x, y, 2, out=pk.token_logprobs_outputs(4, 3)),
           lambda: pk.token_logprobs_grad(x, y, f.double(), f, f), lambda: pk.token_logprobs_grad(x, y, None, f, f),
           lambda: pk.token_logprobs_grad(x, y, f, None, f, f),
           lambda: pk.token_logprobs_grad(x, y, f, f, f, None, y.view(4, 1), f),
           lambda: pk.token_logprobs_grad(x, y, f, f, f, out=x.bfloat16()),
           lambda: pk.token_logprobs_grad(x, y, f, f, f, out=x), lambda: pk.token_logprobs_grad(x, y, f, f, f, out=x.t())]
    for call in bad:
        with pytest.raises(pk.ProfkError):
            call()
