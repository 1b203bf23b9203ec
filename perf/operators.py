"""The operators between a language model's last hidden state and its answer,
and the work they are timed on.

  logprobs   token_logprobs        log probability of a given token per row of
                                   logits, the row's entropy and log-sum-exp,
                                   and its most probable alternatives
  grad       token_logprobs_grad   the gradient of those with respect to the
                                   logits
  quantize   mx4_quantize, mx4_dequantize   values to 4 bits (E2M1) with one
                                   power-of-two scale per 32, and back
  linear     mx4_linear            x W^T with x quantised in the call and W
                                   held in 4 bits

With x one row of V logits, y its token, p = exp(x - lse):

  lse = log sum_j exp(x_j)       logprob = x_y - lse
  entropy H = -sum_j p_j log p_j (terms with p_j = 0 are 0)
  alternatives: the n largest x_j, equal values by smaller index, as
  (x_j - lse, j)

and for gradients g (of logprob), h (of the entropy), t_i (of alternative i,
at index a_i):

  dx_j = g ([j = y] - p_j) - h p_j (log p_j + H) + sum_i t_i ([j = a_i] - p_j)

A block of 32 values v with largest magnitude m > 0 has the scale 2^s, s =
floor(log2 m) - 2 within [-127, 127]; each v / 2^s is rounded to the nearest
of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, larger ones to 6) with
its sign.

listed() holds the sizes of this repository's own configurations, tests and
benchmark and generic ones between them; draw() gives others of the same
ranges.
"""

import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
MAX_LOGITS = 1 << 29        # elements of the largest logits
MAX_PRODUCT = 4096 * 2048 * 131072


def _lp(kind, name, T, V, n_top, dtype, masked=False, pad=0):
    return dict(name=name, kind=kind, T=T, V=V, n_top=n_top, dtype=dtype, masked=masked, pad=pad)


def listed():
    return [
        # One sequence decodes one token: one row, latency.
        _lp("logprobs", "logprobs_f32_1x131072_top20", 1, 131072, 20, "f32"),
        # A decode batch of odd vocabulary, some tokens forbidden.
        _lp("logprobs", "logprobs_f32_64x100003_top20", 64, 100_003, 20, "f32", masked=True),
        # Short rows, many of them: a classifier's or a router's choices.
        _lp("logprobs", "logprobs_f32_16384x512_top8", 16384, 512, 8, "f32"),
        # Scoring a prompt: the per-row configuration, one GiB of logits.
        _lp("logprobs", "logprobs_bf16_4096x131072_top20", 4096, 131072, 20, "bf16"),
        # Training on a batch with an entropy term: one GiB in, one out.
        _lp("grad", "grad_bf16_4096x131072", 4096, 131072, 0, "bf16"),
        # Distillation onto given alternatives, odd vocabulary, padded rows.
        _lp("grad", "grad_f32_509x50001_top16", 509, 50_001, 16, "f32", masked=True, pad=3),
        # The SAE's dictionary to 4 bits.
        dict(name="quantize_bf16_12288x512", kind="quantize", R=12288, K=512, dtype="bf16"),
        # An unembedding to 4 bits, from fp32 master weights.
        dict(name="quantize_f32_131072x2048", kind="quantize", R=131072, K=2048, dtype="f32"),
        # The unembedding for one decoded token: every weight read once.
        dict(name="linear_1x4096x131072_f32", kind="linear", M=1, K=4096, N=131072, dtype="f32"),
        # Ragged sizes: a small batch, a width with a partial block.
        dict(name="linear_77x1000x50001_f32", kind="linear", M=77, K=1000, N=50_001, dtype="f32"),
        # The SAE encoder's product at the paper's shape.
        dict(name="linear_4096x512x12288_f32", kind="linear", M=4096, K=512, N=12288, dtype="f32"),
        # The logits of a prompt.
        dict(name="linear_4096x2048x131072_bf16", kind="linear", M=4096, K=2048, N=131072, dtype="bf16"),
    ]


# ------------------------------------------------------------------ draws ---

def _odd(rng, lo, hi):
    """An odd integer of about lo to hi, spread over its logarithm."""
    return min(int(math.exp(rng.uniform(math.log(lo), math.log(hi)))) | 1, (hi - 1) | 1)


def _size(rng, lo, hi):
    """Odd, or a power of two."""
    if rng.random() < 0.5:
        return _odd(rng, lo, hi)
    return 1 << rng.randint(max(lo - 1, 0).bit_length(), hi.bit_length() - 1)


def draw(rng):
    u = rng.random()
    if u < 0.55:
        kind = "logprobs" if u < 0.35 else "grad"
        dtype = rng.choice(["f32", "bf16"])
        V = _size(rng, 64, 1 << 18)
        T = _size(rng, 1, min((MAX_LOGITS if dtype == "bf16" else MAX_LOGITS // 2) // V, 32768))
        n_top = rng.choice([0, 1, 5, 20, 32]) if kind == "logprobs" else rng.choice([0, 0, 16])
        return dict(kind=kind, T=T, V=V, n_top=n_top, dtype=dtype, masked=rng.random() < 0.4,
                    pad=rng.choice([0, 0, 1, 8]))
    if u < 0.70:
        K = _size(rng, 32, 4096)
        R = _size(rng, 1, min((1 << 28) // K, 1 << 18))
        return dict(kind="quantize", R=R, K=K, dtype=rng.choice(["f32", "bf16"]))
    K = _size(rng, 32, 4096)
    M = _size(rng, 1, 4096)
    N = _size(rng, 64, min(131072, MAX_PRODUCT // (M * K)))
    return dict(kind="linear", M=M, K=K, N=N, dtype=rng.choice(["f32", "bf16"]))


# ----------------------------------------------------------------- inputs ---

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _logits(case, seed):
    """Logits N(0, 2.5), each row with a few likely tokens; masked cases
    forbid three tokens in ten (-inf).  Nine rows in ten are given a token
    that is allowed, the others none (a negative one)."""
    T, V = case["T"], case["V"]
    g = _gen(seed)
    x = torch.randn((T, V + case["pad"]), generator=g, device=DEV)
    x *= 2.5
    likely = torch.randint(V, (T, 8), generator=g, device=DEV)
    # (a value of its column, so that a column drawn twice has one)
    x.scatter_(1, likely, (4.0 + 6.0 * torch.rand(V, generator=g, device=DEV))[likely])
    y = torch.where(torch.rand(T, generator=g, device=DEV) < 0.7, likely[:, 0],
                    torch.randint(V, (T,), generator=g, device=DEV))
    if case["masked"]:
        off = torch.rand(x.shape, generator=g, device=DEV) < 0.3
        off.scatter_(1, likely, False)
        off.scatter_(1, y[:, None], False)
        # (every row allows at least the alternatives asked for)
        off[:, :max(case["n_top"], 1)] = False
        x.masked_fill_(off, -math.inf)
        del off
    y = torch.where(torch.rand(T, generator=g, device=DEV) < 0.9, y, torch.full_like(y, -100))
    return x.to(DTYPE[case["dtype"]])[:, :V], y


def _grad_inputs(case, seed, V):
    g = _gen(seed + 1)
    T, n = case["T"], case["n_top"]
    gl = -torch.rand(T, generator=g, device=DEV)
    gh = 0.1 * torch.randn(T, generator=g, device=DEV)
    gt = -torch.rand((T, n), generator=g, device=DEV) if n else None
    return gl, gh, gt


def _quantize_input(case, seed):
    """Weights, each row of a size of its own, some blocks all zero."""
    g = _gen(seed)
    x = torch.randn((case["R"], case["K"]), generator=g, device=DEV)
    x *= torch.exp(torch.randn((case["R"], 1), generator=g, device=DEV) * 2.0)
    x[torch.rand(case["R"], generator=g, device=DEV) < 0.01] = 0.0
    return x.to(DTYPE[case["dtype"]])


def _linear_inputs(case, seed):
    """Hidden states with a few large channels; weights N(0, 1/K)."""
    g = _gen(seed)
    M, K, N = case["M"], case["K"], case["N"]
    x = torch.randn((M, K), generator=g, device=DEV)
    x[:, ::61] *= 8.0
    w = torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)
    return x.to(torch.bfloat16), w.to(torch.bfloat16)


def prepare(case, seed):
    kind = case["kind"]
    s = dict(kind=kind, case=case)
    if own:
        import paper_2608_12573_amd as pk
    if kind in ("logprobs", "grad"):
        T, V, n = case["T"], case["V"], case["n_top"]
        s["x"], s["y"] = _logits(case, seed)
        if kind == "logprobs":
            if own:
                s["ws"] = pk.token_logprobs_workspace(T, V, n, DEV)
                s["out"] = pk.token_logprobs_outputs(T, n, DEV)
            return s
        # what the forward pass left: the rows' statistics and alternatives
        _, s["h"], s["lse"], _, s["top"] = _plain_logprobs(s["x"], s["y"], n)
        s["gl"], s["gh"], s["gt"] = _grad_inputs(case, seed, V)
        if own:
            s["out"] = torch.empty((T, V), dtype=s["x"].dtype, device=DEV)
        return s
    if kind == "quantize":
        s["x"] = _quantize_input(case, seed)
        if own:
            s["q"] = pk.mx4_outputs(case["R"], case["K"], DEV)
            s["out"] = torch.empty((case["R"], case["K"]), dtype=torch.bfloat16, device=DEV)
        return s
    s["x"], w = _linear_inputs(case, seed)
    if own:
        # the weights are quantised once, as a serving program does
        s["w"] = pk.mx4_quantize(w)
        s["ws"] = pk.mx4_linear_workspace(case["M"], case["K"], case["N"], DEV)
        s["out"] = torch.empty((case["M"], case["N"]), dtype=DTYPE[case["dtype"]], device=DEV)
    else:
        s["w"] = _plain_mx4(w).to(torch.bfloat16)      # (the values are exact in bf16)
    return s


# ------------------------------------------------------------ plain forms ---

def _order(x):
    """An integer per value that orders as the value does, -0 below +0."""
    b = x.contiguous().view(torch.int32)
    return torch.where(b < 0, -(b & 0x7FFFFFFF) - 1, b)


def _plain_rows(x, y, n):
    x = x.float()
    V = x.shape[1]
    m = x.max(dim=1, keepdim=True).values
    d = x - m
    e = torch.exp(d)
    s = e.sum(dim=1, keepdim=True)
    h = torch.log(s) - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(dim=1, keepdim=True) / s
    lse = m + torch.log(s)
    given = (y >= 0) & (y < V)
    lp = torch.where(given, x.gather(1, y.clamp(0, V - 1)[:, None])[:, 0] - lse[:, 0], torch.zeros_like(lse[:, 0]))
    if not n:
        return lp, h[:, 0], lse[:, 0], None, None
    low = (1 << 31) - 1 - torch.arange(V, device=x.device)
    c = _order(x).to(torch.int64) * (1 << 31) + low
    top = (1 << 31) - 1 - (torch.topk(c, n, dim=1).values & ((1 << 31) - 1))
    return lp, h[:, 0], lse[:, 0], x.gather(1, top) - lse, top


def _plain_logprobs(x, y, n):
    step = max(1, (1 << 27) // x.shape[1])
    parts = [_plain_rows(x[r:r + step], y[r:r + step], n) for r in range(0, x.shape[0], step)]
    return tuple(torch.cat(c) if c[0] is not None else None for c in zip(*parts))


def _plain_grad(s):
    x, out = s["x"], []
    V = x.shape[1]
    step = max(1, (1 << 27) // V)
    for r in range(0, x.shape[0], step):
        part = slice(r, r + step)
        y, gh, h = s["y"][part, None], s["gh"][part, None], s["h"][part, None]
        given = (y >= 0) & (y < V)
        gl = torch.where(given, s["gl"][part, None], torch.zeros_like(gh))
        total = gl if s["gt"] is None else gl + s["gt"][part].sum(dim=1, keepdim=True)
        l = x[part].float() - s["lse"][part, None]
        p = torch.exp(l)
        d = torch.where(p > 0, -p * (total + gh * (l + h)), torch.zeros_like(p))
        d.scatter_add_(1, y.clamp(0, V - 1), gl)
        if s["gt"] is not None:
            d.scatter_add_(1, s["top"][part], s["gt"][part])
        out.append(d.to(x.dtype))
    return torch.cat(out)


def _pow2(e):
    """2^e as two fp32 factors, each exact (a power function's last bit need
    not be)."""
    half = torch.div(e, 2, rounding_mode="floor")
    return [((h + 127).to(torch.int32) << 23).view(torch.float32) for h in (half, e - half)]


def _plain_mx4(x):
    """The values that x's 4-bit form stands for, fp32."""
    R, K = x.shape
    v = torch.nn.functional.pad(x.float(), (0, -K % 32)).view(R, -1, 32)
    m = v.abs().amax(dim=2, keepdim=True)
    e = (torch.frexp(m).exponent - 3).clamp(-127, 127)
    up, down = _pow2(e), _pow2(-e)
    a = v.abs() * down[0] * down[1]
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    q = torch.clamp(torch.round(a / step) * step, max=6.0) * up[0] * up[1]
    return torch.copysign(q, v).reshape(R, -1)[:, :K]


def run(s):
    kind, case = s["kind"], s["case"]
    if own:
        import paper_2608_12573_amd as pk
        if kind == "logprobs":
            out = pk.token_logprobs(s["x"], s["y"], case["n_top"], ws=s["ws"], out=s["out"])
            return out if case["n_top"] else out[:3]
        if kind == "grad":
            return pk.token_logprobs_grad(s["x"], s["y"], s["lse"], s["h"], s["gl"], s["gh"], s["top"], s["gt"],
                                          out=s["out"])
        if kind == "quantize":
            codes, scales = pk.mx4_quantize(s["x"], out=s["q"])
            return pk.mx4_dequantize(codes, scales, case["K"], out=s["out"])
        return pk.mx4_linear(s["x"], *s["w"], ws=s["ws"], out=s["out"])
    if kind == "logprobs":
        out = _plain_logprobs(s["x"], s["y"], case["n_top"])
        return out if case["n_top"] else out[:3]
    if kind == "grad":
        return _plain_grad(s)
    if kind == "quantize":
        return _plain_mx4(s["x"]).to(torch.bfloat16)
    return (_plain_mx4(s["x"]) @ s["w"].float().t()).to(DTYPE[case["dtype"]])


def work(case):
    kind = case["kind"]
    if kind in ("logprobs", "grad"):
        n, T, n_top = case["T"] * case["V"], case["T"], case["n_top"]
        es = BYTES[case["dtype"]]
        if kind == "logprobs":   # logits and tokens; three numbers and the alternatives
            return {"bytes": n * es + T * (8 + 12) + T * n_top * 12, "flops": 5 * n}
        return {"bytes": 2 * n * es + T * (8 + 16) + T * n_top * 12, "flops": 5 * n}
    if kind == "quantize":       # values in, codes and scales out and in, values out
        blocks = case["R"] * -(-case["K"] // 32)
        return {"bytes": case["R"] * case["K"] * (BYTES[case["dtype"]] + 2) + 2 * 17 * blocks,
                "flops": 2 * case["R"] * case["K"]}
    M, K, N = case["M"], case["K"], case["N"]
    return {"bytes": M * K * 2 + N * -(-K // 32) * 17 + M * N * BYTES[case["dtype"]], "flops": 2 * M * K * N}


# ------------------------------------------------------------- in 64 bits ---

def _exact_logprobs(x, y, n):
    out = []
    step = max(1, (1 << 26) // x.shape[1])
    for r in range(0, x.shape[0], step):
        z = x[r:r + step].double()
        t = y[r:r + step]
        lse = torch.logsumexp(z, dim=1)
        l = z - lse[:, None]
        h = -torch.special.xlogy(l.exp(), l.exp()).sum(dim=1)
        lp = torch.where(t < 0, 0.0, l.gather(1, t.clamp(min=0)[:, None])[:, 0])
        alt_l, alt_j = [], []
        col = torch.arange(z.shape[1], device=z.device)
        for _ in range(n):   # the largest left, at its first place
            best = z.amax(dim=1, keepdim=True)
            j = torch.where(z == best, col, z.shape[1]).amin(dim=1, keepdim=True)
            alt_l.append(l.gather(1, j))
            alt_j.append(j)
            z.scatter_(1, j, -math.inf)
        out.append((lp, h, lse) + ((torch.cat(alt_l, 1), torch.cat(alt_j, 1)) if n else ()))
    return tuple(torch.cat(c) for c in zip(*out))


def _exact_grad(case, seed):
    x, y = _logits(case, seed)
    n, V = case["n_top"], case["V"]
    gl, gh, gt = _grad_inputs(case, seed, V)
    top = _plain_logprobs(x, y, n)[4] if n else None
    out = torch.empty(x.shape, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // V)
    for r in range(0, x.shape[0], step):
        z = x[r:r + step].double()
        l = z - torch.logsumexp(z, dim=1, keepdim=True)
        p = l.exp()
        # upstream gradient of every log probability, then the softmax's
        # Jacobian; H = -sum p log p adds -h (log p + 1) p through dp
        u = torch.zeros_like(z)
        t = y[r:r + step]
        u.scatter_(1, t.clamp(min=0)[:, None], torch.where(t < 0, 0.0, gl[r:r + step].double())[:, None])
        if n:
            u.scatter_add_(1, top[r:r + step], gt[r:r + step].double())
        u -= gh[r:r + step, None].double() * (p + torch.special.xlogy(p, p))
        out[r:r + step] = u - p * u.sum(dim=1, keepdim=True)
    return out


def _exact_mx4(x):
    """The nearest representable value of every element, by comparison with
    the midpoints between neighbours."""
    R, K = x.shape
    out = torch.zeros((R, -(-K // 32) * 32), dtype=torch.float64, device=x.device)
    out[:, :K] = x
    v = out.view(R, -1, 32)
    m = v.abs().amax(dim=2, keepdim=True)
    s = (((m.view(torch.int64) >> 52) - 1023) - 2).double()     # (fp32 values are normal in 64 bits)
    unit = ((s.clamp(-127, 127) + 1023).to(torch.int64) << 52).view(torch.float64)
    a = v.abs() / unit
    grid = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
    q = torch.zeros_like(a)
    for i in range(1, 8):
        mid = (grid[i - 1] + grid[i]) / 2
        # an even code takes the midpoint below it
        q = torch.where(a >= mid if i % 2 == 0 else a > mid, grid[i], q)
    return torch.where(m > 0, q * unit * torch.sign(v), 0.0).view(R, -1)[:, :K]


def exact(case, seed):
    kind = case["kind"]
    if kind == "logprobs":
        return _exact_logprobs(*_logits(case, seed), case["n_top"])
    if kind == "grad":
        return _exact_grad(case, seed)
    if kind == "quantize":
        return _exact_mx4(_quantize_input(case, seed))
    x, w = _linear_inputs(case, seed)
    a = _exact_mx4(x)
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=DEV)
    for c in range(0, case["N"], 16384):
        out[:, c:c + 16384] = a @ _exact_mx4(w[c:c + 16384]).t()
    return out
