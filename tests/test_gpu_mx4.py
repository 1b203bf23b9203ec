"""4-bit microscaled quantisation and product on the GPU against the oracle.

Codes, scales and dequantised values are exact.  The product's terms are exact
too (2-bit significands times powers of two); the matrix cores round the sum
of 64 of them and the accumulator once a step.  With s the sum of the terms'
magnitudes, an fp32 result is off by at most (K / 64 + 2) 2^-23 s (one ulp a
step, whether it rounds or truncates); bf16 rounds it once more to 8 bits."""

import numpy as np
import pytest

import paper_2608_12573_amd as pk
from oracle import mx4 as omx
from gpu_util import note, torch

pytestmark = pytest.mark.gpu


def _rows(x, dtype, pad=0, offset=0):
    t = torch()
    R, K = x.shape
    dt = t.float32 if dtype == "f32" else t.bfloat16
    big = t.full((offset + R * (K + pad),), float("nan"), dtype=dt, device="cuda")
    g = big[offset:].view(R, K + pad)[:, :K]
    g.copy_(t.from_numpy(np.ascontiguousarray(x)).cuda().to(dt))
    return g, g.double().cpu().numpy()


def _x(R, K, seed, spread=2.0):
    g = np.random.default_rng(seed)
    x = g.standard_normal((R, K)) * np.exp(g.standard_normal((R, 1)) * spread)
    x[g.random(R) < 0.1] = 0.0
    return x.astype(np.float32)


def _same_values(got, ref):
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    ok = ~np.isnan(ref)
    assert np.array_equal(got[ok], ref[ok])


def _check_quantize(x, dtype, pad=0, offset=0):
    t = torch()
    R, K = x.shape
    note(f"mx4 quantize {dtype} R={R} K={K} pad={pad} offset={offset}")
    g, v = _rows(x, dtype, pad, offset)
    codes, scales = pk.mx4_quantize(g)
    code, byte = omx.quantize(v)
    # [R / 32, Kp / 128, 32, 4]: rows in groups of 32, the last one's rest 0
    groups = -(-R // 32)
    got = scales.cpu().numpy().transpose(0, 2, 1, 3).reshape(groups * 32, -1)
    assert np.array_equal(got[:R], byte.astype(np.uint8)) and not got[R:].any()
    got, ref = codes.cpu().numpy(), omx.pack(code)
    # (codes of a NaN block have no meaning)
    ok = np.repeat(byte != 255, 16, axis=1)
    assert np.array_equal(got[ok], ref[ok])
    val = omx.values(code, byte, K)
    for dt in (t.bfloat16, t.float32):
        _same_values(pk.mx4_dequantize(codes, scales, K, dt).double().cpu().numpy(), val)


@pytest.mark.parametrize("R,K", [(1, 1), (3, 31), (2, 32), (5, 33), (4, 127), (7, 128), (3, 129), (9, 512), (17, 1000),
                                 (2, 4099), (1, 70001), (300, 256), (1000, 65)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_sizes(R, K, dtype):
    _check_quantize(_x(R, K, R + K), dtype)


@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (8, 3), (5, 7)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_strides(pad, offset, dtype):
    _check_quantize(_x(11, 203, 1), dtype, pad, offset)


def test_quantize_every_rounding():
    """Every bf16 magnitude of a few binades against a block of each scale:
    ties, saturation, subnormals, the smallest and largest scales."""
    bits = np.arange(0x0000, 0x7F80, 1, dtype=np.uint32)          # all finite bf16 magnitudes
    v = (bits << 16).view(np.float32).astype(np.float32)
    g = np.random.default_rng(0)
    rows = []
    for top in (2.0 ** -149, 2.0 ** -130, 2.0 ** -126, 1.5 * 2.0 ** -125, 2.0 ** -124, 2.0 ** -123, 2.0 ** -100, 2.0 ** -64,
                2.0 ** -62, 2.0 ** -60, 1.0, 1.75, 2.0 ** 60, 2.0 ** 100, 2.0 ** 127, float(np.finfo(np.float32).max)):
        m = int(np.float32(top).view(np.uint32))
        near = v[(v <= np.float32(top)) & (v >= np.float32(top) * np.float32(2.0 ** -6))]
        near = np.concatenate([near, v[:256], np.zeros(31 - (near.size + 255) % 31, np.float32)])
        near = near[:near.size // 31 * 31].reshape(-1, 31)
        near = np.where(near > np.float32(top), np.float32(0), near)
        near *= np.where(g.random(near.shape) < 0.5, np.float32(-1), np.float32(1))
        rows.append(np.concatenate([np.full((near.shape[0], 1), np.uint32(m).view(np.float32)), near], axis=1))
    x = np.concatenate(rows).astype(np.float32)
    _check_quantize(x, "f32")
    _check_quantize(x[(x[:, 0] > 1e-37) & (x[:, 0] < 1e38)], "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_infinities_and_nan(dtype):
    x = _x(6, 300, 4)
    x[0, 5] = np.inf
    x[1, 40] = -np.inf
    x[2, 299] = np.nan
    x[3] = -0.0
    _check_quantize(x, dtype)


def _pair(M, N, K, seed):
    """Quantised operands and their exact product in fp64."""
    t = torch()
    a, b = _x(M, K, seed, 0.5), _x(N, K, seed + 1, 0.5)
    ga, gb = t.from_numpy(a).cuda(), t.from_numpy(b).cuda()
    qa, qb = pk.mx4_quantize(ga), pk.mx4_quantize(gb)
    va, vb = omx.round_trip(a), omx.round_trip(b)
    return ga, qa, qb, va @ vb.T, np.abs(va) @ np.abs(vb).T


SIZES = [(1, 1, 1), (1, 7, 33), (2, 64, 32), (3, 129, 128), (1, 1000, 4096), (17, 255, 257), (31, 33, 512), (33, 513, 640),
         (64, 64, 1000), (77, 501, 1000), (127, 130, 384), (128, 128, 128), (129, 257, 129), (255, 511, 896),
         (256, 256, 256), (300, 700, 2048), (513, 1025, 768), (1000, 37, 1500), (5, 70001, 300),
         (20, 300, 2048), (32, 1001, 3001), (3, 40000, 1000), (1, 140001, 130), (600, 30000, 512), (1025, 33001, 300)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_product_sizes(M, N, K):
    t = torch()
    note(f"mx4 product M={M} N={N} K={K}")
    x, qa, qb, ref, scale = _pair(M, N, K, M + N + K)
    tol = (K / 64 + 2) * 2.0 ** -23 * scale
    f = pk.mx4_matmul(*qa, *qb, K)
    err = np.abs(f.double().cpu().numpy() - ref)
    assert (err <= tol).all(), (err - tol).max()
    h = pk.mx4_matmul(*qa, *qb, K, t.bfloat16)
    assert t.equal(h, f.bfloat16())
    # from fp32 activations quantised in the call: the same product
    assert t.equal(pk.mx4_linear(x, *qb), f)
    assert t.equal(pk.mx4_linear(x, *qb, dtype=t.bfloat16), h)


def test_linear_of_strided_bf16():
    t = torch()
    note("mx4 linear strided bf16")
    x, v = _rows(_x(9, 203, 3, 0.5), "bf16", 5, 3)
    w = _x(45, 203, 5, 0.5)
    q = pk.mx4_quantize(t.from_numpy(w).cuda())
    a, b = omx.round_trip(v), omx.round_trip(w)
    got = pk.mx4_linear(x, *q).double().cpu().numpy()
    assert (np.abs(got - a @ b.T) <= 6 * 2.0 ** -23 * (np.abs(a) @ np.abs(b).T)).all()


def test_product_of_extreme_scales():
    """Scales from the smallest to the largest on either side: results in
    range are exact, those past it are infinite, those below it vanish."""
    t = torch()
    note("mx4 product, extreme scales")
    e = np.array([-127, -126, -100, -64, -1, 0, 1, 64, 100, 120, 125])
    a = np.zeros((e.size, 128), dtype=np.float32)
    a[:, 0] = np.ldexp(1.0, e).astype(np.float32)
    q = pk.mx4_quantize(t.from_numpy(a).cuda())
    got = pk.mx4_matmul(*q, *q, 128).double().cpu().numpy()
    with np.errstate(over="ignore"):
        ref = (a.astype(np.float64)[:, :1] * a.astype(np.float64)[:, 0]).astype(np.float32).astype(np.float64)
    normal = np.abs(ref) >= 2.0 ** -126
    assert np.array_equal(got[normal], ref[normal])
    assert (np.abs(got[~normal]) <= 2.0 ** -126).all()    # (subnormal sums may be flushed)


def test_product_of_nan_blocks():
    t = torch()
    note("mx4 product with NaN blocks")
    x = _x(40, 300, 1, 0.5)
    w = _x(50, 300, 2, 0.5)
    x[x == 0] = 1.0
    x[3, 100] = np.inf
    w[7, 299] = np.nan
    q = pk.mx4_quantize(t.from_numpy(w).cuda())
    got = pk.mx4_linear(t.from_numpy(x).cuda(), *q).cpu().numpy()
    nan = np.zeros((40, 50), dtype=bool)
    nan[3] = True
    nan[:, 7] = True
    assert np.array_equal(np.isnan(got), nan)


def test_quantize_past_32_bit_offsets():
    t = torch()
    R, K, stride = 3, 1001, (1 << 31) + 9
    big = t.empty(2 * stride + K, dtype=t.bfloat16, device="cuda")
    g = big.as_strided((R, K), (stride, 1))
    g.copy_(t.from_numpy(_x(R, K, 3)).cuda().to(t.bfloat16))
    note("mx4 quantize at 64-bit offsets")
    a, b = pk.mx4_quantize(g), pk.mx4_quantize(g.contiguous())
    assert t.equal(a[0], b[0]) and t.equal(a[1], b[1])


def test_product_past_32_bit_offsets():
    """An output of more than 2^32 bytes, its last rows against the same rows
    alone."""
    t = torch()
    M, N, K = 2051, 1 << 20, 65
    note("mx4 product, output past 4 GiB")
    g = t.Generator(device="cuda").manual_seed(0)
    x = t.randn((M, K), generator=g, device="cuda")
    q = pk.mx4_quantize(t.randn((N, K), generator=g, device="cuda"))
    out = pk.mx4_linear(x, *q, dtype=t.bfloat16)
    assert t.equal(out[-3:], pk.mx4_linear(x[-3:], *q, dtype=t.bfloat16))


def test_no_rows():
    t = torch()
    e = t.empty((0, 70), device="cuda")
    q = pk.mx4_quantize(e)
    assert q[0].shape == (0, 64) and q[1].shape == (0, 1, 32, 4)
    assert pk.mx4_dequantize(*q, 70).shape == (0, 70)
    w = pk.mx4_quantize(t.ones((5, 70), device="cuda"))
    assert pk.mx4_linear(e, *w).shape == (0, 5)
    assert pk.mx4_matmul(*w, *q, 70).shape == (5, 0)


def test_side_stream_and_kept_buffers():
    t = torch()
    M, K, N = 40, 520, 300
    w = t.from_numpy(_x(N, K, 5, 0.5)).cuda()
    xs = [t.from_numpy(_x(M, K, s, 0.5)).cuda() for s in (1, 2)]
    q = pk.mx4_quantize(w)
    ws, out = pk.mx4_linear_workspace(M, K, N), t.empty((M, N), device="cuda")
    ref = [pk.mx4_linear(x, *q) for x in xs]
    note("mx4 linear on a side stream")
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        first = pk.mx4_linear(xs[0], *q, ws=ws, out=out).clone()
        pk.mx4_linear(xs[1], *q, ws=ws, out=out)
    side.synchronize()
    assert t.equal(first, ref[0]) and t.equal(out, ref[1])


@pytest.mark.parametrize("M", [3, 200])
def test_graph_replays(M):
    t = torch()
    K, N = 520, 300
    x = t.from_numpy(_x(M, K, 1, 0.5)).cuda()
    q = pk.mx4_quantize(t.from_numpy(_x(N, K, 5, 0.5)).cuda())
    ws, out = pk.mx4_linear_workspace(M, K, N), t.empty((M, N), device="cuda")
    note(f"mx4 linear under capture M={M}")
    ref = pk.mx4_linear(x, *q, ws=ws, out=out).clone()
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        pk.mx4_linear(x, *q, ws=ws, out=out)
    t.cuda.current_stream().wait_stream(side)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        pk.mx4_linear(x, *q, ws=ws, out=out)
    for _ in range(3):
        out.fill_(-7)
        ws.fill_(255)
        t.cuda.synchronize()
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(out, ref)


def test_refusals_on_the_device():
    t = torch()
    x = t.zeros(4, 64, device="cuda")
    c, s = pk.mx4_quantize(x)
    bad = [lambda: pk.mx4_quantize(x, out=pk.mx4_outputs(5, 64)), lambda: pk.mx4_quantize(x, out=pk.mx4_outputs(4, 129)),
           lambda: pk.mx4_dequantize(c, s[:, :, :3], 64), lambda: pk.mx4_dequantize(c, s, 64, t.float16),
           lambda: pk.mx4_dequantize(c, s.cpu(), 64), lambda: pk.mx4_matmul(c, s, c, s, 129),
           lambda: pk.mx4_matmul(c, s, c, s, 64, out=t.zeros(4, 5, device="cuda")),
           lambda: pk.mx4_linear(x, c, s, ws=t.zeros(8, dtype=t.uint8)),
           lambda: pk.mx4_linear(x, c, s, dtype=t.bfloat16, out=t.zeros(4, 4, device="cuda")),
           lambda: pk.mx4_linear(t.zeros(4, 200, device="cuda"), c, s)]
    for call in bad:
        with pytest.raises(pk.ProfkError):
            call()


def test_output_refusals():
    t = torch()
    x = t.ones(4, 100, device="cuda")
    q = pk.mx4_quantize(x)
    for out, dtype, match in (([0.0], t.float32, "torch tensor"), ([0.0], None, "torch tensor"),
                              (t.empty(4, 4, device="cuda"), t.bfloat16, "not torch.bfloat16"),
                              (t.empty(4, 5, device="cuda"), None, "shape"),
                              (t.empty(4, 4), None, "CUDA tensor"),
                              (t.empty(4, 4, device="cuda").half(), None, "unsupported dtype")):
        print(match, dtype, flush=True)
        for call in (lambda: pk.mx4_matmul(*q, *q, 100, dtype=dtype, out=out),
                     lambda: pk.mx4_linear(x, *q, dtype=dtype, out=out)):
            with pytest.raises(pk.ProfkError, match=match):
                call()
    with pytest.raises(pk.ProfkError, match="4 rows"):
        pk.mx4_quantize(x, out=pk.mx4_outputs(5, 100, "cuda"))
