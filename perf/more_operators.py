"""Normalisation, dense product and penalties: the operators before and after
a row of logits, and the work they are timed on.

  norm         layer_norm           rows normalised to mean 0 and variance 1,
                                    scaled and shifted
  norm_grad    layer_norm_grad      its gradients: of the rows, the scale and
                                    the shift
  linear       linear               act(x W^T + b) + residual
  linear_grad  linear_grad          its gradients: of x, W and b
  adjust       adjust_logits        penalties for repeated tokens, biases and
                                    masks of allowed tokens on rows of logits
  adjust_grad  adjust_logits_grad   the gradient of those with respect to the
                                    logits

Of one row x of D values, mean m, r = 1 / sqrt(mean (x - m)^2 + eps):

  y = (x - m) r w + b

and with n = (x - m) r and g = dy w:

  dx = r (g - mean g - n mean (g n))    dw = sum over rows dy n
  db = sum over rows dy

Of the product, z = x W^T + b, y = act(z) + residual, dz = dy act'(z):

  dx = dz W    dW = dz^T x    db = sum over rows dz

Of one row of logits x, with its history of tokens, the first n_prompt of them
a prompt, c_v the occurrences of v after the prompt:

  u_v = x_v / repetition if x_v > 0, else x_v * repetition   (v in the history)
  u_v = x_v                                                  (v not in it)
  y_v = u_v - [c_v > 0] presence - c_v frequency + bias_v,   or -inf where the
                                                             row's mask forbids v

and the gradient of x is that of y times 1 / repetition, repetition or 1, and 0
where v is forbidden.

listed() holds sizes of this repository's own configurations, tests and
benchmark and generic ones between them; draw() gives others of the same
ranges.
"""

import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "bf16": 2}
EPS = 1e-5
ACTIVATIONS = [None, "relu", "gelu", "silu"]
MAX_NORM = 16384 * 8192         # elements of the largest normalised matrix
MAX_LOGITS = 4096 * 131072      # ... of the largest logits
MAX_PRODUCT = 4096 * 4096 * 12288


def _norm(kind, name, T, D, dtype, out, pad=0):
    return dict(name=name, kind=kind, T=T, D=D, dtype=dtype, out=out, pad=pad)


def _linear(kind, name, M, K, N, act, out, bias=True, residual=False):
    return dict(name=name, kind=kind, M=M, K=K, N=N, act=act, out=out, bias=bias, residual=residual)


def _adjust(kind, name, T, V, dtype, history, masks, biases, pad=0):
    return dict(name=name, kind=kind, T=T, V=V, dtype=dtype, history=history, masks=masks, biases=biases, pad=pad)


def listed():
    return [
        # The last norm of one decoded token: latency.
        _norm("norm", "norm_bf16_1x4096", 1, 4096, "bf16", "bf16"),
        # The norm of a long prompt's hidden states.
        _norm("norm", "norm_bf16_16384x8192", 16384, 8192, "bf16", "bf16"),
        # Odd rows with a gap between them, fp32 in training.
        _norm("norm_grad", "norm_grad_f32_2047x1001", 2047, 1001, "f32", "f32", pad=3),
        # The norm's backward pass over a training batch.
        _norm("norm_grad", "norm_grad_bf16_16384x4096", 16384, 4096, "bf16", "bf16"),
        # One decoded token through a wide layer: every weight read once.
        _linear("linear", "linear_1x4096x12288_gelu", 1, 4096, 12288, "gelu", "bf16"),
        # A prompt through it, the residual stream added.
        _linear("linear", "linear_4096x4096x12288_silu", 4096, 4096, 12288, "silu", "bf16", residual=True),
        # Odd sizes, as a probe or a small head is trained.
        _linear("linear_grad", "linear_grad_509x1001x777_relu", 509, 1001, 777, "relu", "f32"),
        # The backward pass of a layer over a training batch.
        _linear("linear_grad", "linear_grad_4096x2048x12288_gelu", 4096, 2048, 12288, "gelu", "bf16"),
        # One sequence decodes: a history, a grammar, some biases.
        _adjust("adjust", "adjust_f32_1x131072", 1, 131072, "f32", 1024, 1, 16),
        # A decode batch of long histories, half of it under a grammar.
        _adjust("adjust", "adjust_bf16_256x131072", 256, 131072, "bf16", 4096, 8, 32),
        # Training on tokens that were sampled under penalties, odd vocabulary.
        _adjust("adjust_grad", "adjust_grad_f32_509x50001", 509, 50_001, "f32", 512, 4, 0, pad=3),
        # The same over a batch of whole sequences.
        _adjust("adjust_grad", "adjust_grad_bf16_4096x131072", 4096, 131072, "bf16", 256, 0, 0),
    ]


# ------------------------------------------------------------------ draws ---

def _odd(rng, lo, hi):
    """An odd integer of about lo to hi, spread over its logarithm."""
    return min(int(math.exp(rng.uniform(math.log(lo), math.log(hi)))) | 1, (hi - 1) | 1)


def _size(rng, lo, hi):
    """Odd, a multiple of eight, or a power of two."""
    u = rng.random()
    if u < 0.4 or hi < 16:
        return max(lo, min(_odd(rng, lo, hi + 1), hi))
    if u < 0.7:
        return max(8, min(_odd(rng, max(lo, 8), hi) // 8 * 8, hi // 8 * 8))
    return 1 << rng.randint(max(lo - 1, 0).bit_length(), hi.bit_length() - 1)


def draw(rng):
    u = rng.random()
    if u < 0.35:
        kind = "norm" if u < 0.17 else "norm_grad"
        D = _size(rng, 16, 16384)
        T = _size(rng, 1, min(MAX_NORM // 2 // D, 65536))
        dtype = rng.choice(["f32", "bf16"])
        return dict(kind=kind, T=T, D=D, dtype=dtype, out=rng.choice([dtype, "bf16"]), pad=rng.choice([0, 0, 1, 8]))
    if u < 0.7:
        kind = "linear" if u < 0.55 else "linear_grad"
        K = _size(rng, 16, 8192)
        M = _size(rng, 1, 8192)
        N = _size(rng, 16, max(16, min(16384, MAX_PRODUCT // (2 * M * K))))
        return dict(kind=kind, M=M, K=K, N=N, act=rng.choice(ACTIVATIONS), out=rng.choice(["f32", "bf16"]),
                    bias=rng.random() < 0.7, residual=kind == "linear" and rng.random() < 0.4)
    kind = "adjust" if u < 0.87 else "adjust_grad"
    dtype = rng.choice(["f32", "bf16"])
    V = _size(rng, 64, 1 << 18)
    T = _size(rng, 1, min((MAX_LOGITS if dtype == "bf16" else MAX_LOGITS // 2) // V, 8192))
    return dict(kind=kind, T=T, V=V, dtype=dtype, history=_odd(rng, 1, min(8192, max(3, (1 << 22) // T))),
                masks=rng.choice([0, 1, 5]), biases=rng.choice([0, 0, 3, 50]) if kind == "adjust" else 0,
                pad=rng.choice([0, 0, 1, 8]))


# ----------------------------------------------------------------- inputs ---

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _norm_inputs(case, seed):
    """Hidden states: rows of their own size and mean, a few large channels;
    a scale near 1, a small shift; the gradient of the output."""
    g = _gen(seed)
    T, D = case["T"], case["D"]
    x = torch.randn((T, D + case["pad"]), generator=g, device=DEV)
    x[:, ::61] *= 8.0
    x *= torch.exp(0.5 * torch.randn((T, 1), generator=g, device=DEV))
    x += 0.3 * torch.randn((T, 1), generator=g, device=DEV)
    w = 1.0 + 0.2 * torch.randn(D, generator=g, device=DEV)
    b = 0.1 * torch.randn(D, generator=g, device=DEV)
    dy = torch.randn((T, D), generator=g, device=DEV) if case["kind"] == "norm_grad" else None
    return x.to(DTYPE[case["dtype"]])[:, :D], w, b, None if dy is None else dy.to(DTYPE[case["out"]])


def _linear_inputs(case, seed):
    """Hidden states with a few large channels; weights N(0, 1/K); fp32
    biases; a residual stream or the gradient of the output."""
    g = _gen(seed)
    M, K, N = case["M"], case["K"], case["N"]
    x = torch.randn((M, K), generator=g, device=DEV)
    x[:, ::61] *= 8.0
    w = torch.randn((N, K), generator=g, device=DEV) / math.sqrt(K)
    b = 0.1 * torch.randn(N, generator=g, device=DEV) if case["bias"] else None
    r = None
    if case["residual"] or case["kind"] == "linear_grad":
        r = torch.randn((M, N), generator=g, device=DEV).to(DTYPE[case["out"]])
    return x.to(torch.bfloat16), w.to(torch.bfloat16), b, r


def _adjust_inputs(case, seed):
    """Logits N(0, 2.5); histories of half to all of the given length, some
    empty, drawn mostly from a few hundred tokens so that they repeat; a third
    of each is the prompt.  Masks allow a tenth of the tokens; half of the rows
    have one.  Rows' penalties are of the sizes that are offered to users."""
    g = _gen(seed)
    T, V, L = case["T"], case["V"], case["history"]
    x = (2.5 * torch.randn((T, V + case["pad"]), generator=g, device=DEV)).to(DTYPE[case["dtype"]])[:, :V]
    n = torch.randint(L // 2, L + 1, (T,), generator=g, device=DEV)
    n = torch.where(torch.rand(T, generator=g, device=DEV) < 0.05, torch.zeros_like(n), n)
    offsets = torch.zeros(T + 1, dtype=torch.int64, device=DEV)
    offsets[1:] = torch.cumsum(n, 0)
    total = int(offsets[-1])
    common = torch.randint(V, (512,), generator=g, device=DEV)
    tokens = torch.where(torch.rand(total, generator=g, device=DEV) < 0.7,
                         common[torch.randint(512, (total,), generator=g, device=DEV)],
                         torch.randint(V, (total,), generator=g, device=DEV))
    s = dict(x=x, tokens=tokens, offsets=offsets, n_prompt=n // 3,
             repetition=1.0 + 0.5 * torch.rand(T, generator=g, device=DEV),
             presence=torch.rand(T, generator=g, device=DEV), frequency=0.5 * torch.rand(T, generator=g, device=DEV),
             bias=None, allowed=None, mask=None)
    if case["biases"]:
        k = case["biases"]
        # distinct tokens of a row: one from each of k parts of the vocabulary
        part = torch.arange(k, device=DEV) * (V // k)
        ids = part + torch.randint(max(V // k, 1), (T, k), generator=g, device=DEV)
        s["bias"] = (ids.reshape(-1), 4.0 * torch.randn(T * k, generator=g, device=DEV),
                     torch.arange(T + 1, device=DEV) * k)
    if case["masks"]:
        words = -(-V // 32)
        bits = (torch.rand((case["masks"], words, 32), generator=g, device=DEV) < 0.1).to(torch.int64)
        packed = (bits << torch.arange(32, device=DEV)).sum(dim=2)
        s["allowed"] = torch.where(packed >= 1 << 31, packed - (1 << 32), packed).to(torch.int32)
        mask = torch.randint(case["masks"], (T,), generator=g, device=DEV)
        s["mask"] = torch.where(torch.rand(T, generator=g, device=DEV) < 0.5, mask, torch.full_like(mask, -1))
    if case["kind"] == "adjust_grad":
        # the gradient of log probabilities: most of a row's is small
        dy = torch.randn((T, V), generator=g, device=DEV)
        s["dy"] = (dy * dy * dy * 1e-2).to(DTYPE[case["dtype"]])
    return s


def prepare(case, seed):
    kind = case["kind"]
    s = dict(kind=kind, case=case)
    if own:
        import paper_2608_12573_amd as pk
    if kind in ("norm", "norm_grad"):
        T, D = case["T"], case["D"]
        s["x"], s["w"], s["b"], s["dy"] = _norm_inputs(case, seed)
        if kind == "norm":
            if own:
                s["out"] = pk.layer_norm_outputs(T, D, DTYPE[case["out"]], DEV)
            return s
        # what the forward pass left
        _, s["mean"], s["rstd"] = _plain_norm(s["x"], s["w"], s["b"], torch.float32)
        if own:
            s["ws"] = pk.layer_norm_grad_workspace(T, D, DEV)
            s["out"] = (torch.empty((T, D), dtype=s["x"].dtype, device=DEV), torch.empty(D, device=DEV),
                        torch.empty(D, device=DEV))
        return s
    if kind in ("linear", "linear_grad"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"], s["w"], s["b"], s["r"] = _linear_inputs(case, seed)
        if kind == "linear":
            if own:
                s["ws"] = pk.linear_workspace(M, K, N, DEV)
                s["out"] = torch.empty((M, N), dtype=DTYPE[case["out"]], device=DEV)
            return s
        # what the forward pass kept
        s["z"] = _plain_product(s["x"], s["w"], s["b"]).to(DTYPE[case["out"]])
        if own:
            s["ws"] = pk.linear_grad_workspace(M, K, N, DEV)
            s["out"] = (torch.empty((M, K), dtype=torch.bfloat16, device=DEV),
                        torch.empty((N, K), dtype=torch.bfloat16, device=DEV), torch.empty(N, device=DEV))
        return s
    s.update(_adjust_inputs(case, seed))
    if own:
        s["out"] = torch.empty((case["T"], case["V"]), dtype=s["x"].dtype, device=DEV)
    else:
        s["edges"] = s["offsets"].tolist()
    return s


# ------------------------------------------------------------ plain forms ---

def _plain_norm(x, w, b, dtype):
    x = x.float()
    m = x.mean(dim=1, keepdim=True)
    c = x - m
    r = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + EPS)
    return (c * r * w + b).to(dtype), m[:, 0], r[:, 0]


def _plain_norm_grad(s):
    x, dy = s["x"].float(), s["dy"].float()
    r = s["rstd"][:, None]
    n = (x - s["mean"][:, None]) * r
    g = dy * s["w"]
    dx = r * (g - g.mean(dim=1, keepdim=True) - n * (g * n).mean(dim=1, keepdim=True))
    return dx.to(s["x"].dtype), (dy * n).sum(dim=0), dy.sum(dim=0)


def _plain_product(x, w, b):
    z = x.float() @ w.float().t()
    return z if b is None else z + b


def _plain_act(z, act):
    if act == "relu":
        return torch.clamp(z, min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _plain_slope(z, act):
    if act == "relu":
        return (z > 0).float()
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _plain_linear(s):
    y = _plain_act(_plain_product(s["x"], s["w"], s["b"]), s["case"]["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(DTYPE[s["case"]["out"]])


def _plain_linear_grad(s):
    dz = s["r"].float() * _plain_slope(s["z"].float(), s["case"]["act"])
    return ((dz @ s["w"].float()).to(torch.bfloat16), (dz.t() @ s["x"].float()).to(torch.bfloat16), dz.sum(dim=0))


def _plain_rows_of(offsets, lo, hi, first, last):
    """The rows, from `first` up, of the entries lo..hi of a ragged list."""
    at = torch.arange(lo, hi, device=DEV)
    return torch.searchsorted(offsets[first + 1:last + 1].contiguous(), at, right=True), at


def _plain_seen(s, first, last, V):
    """Counts of each token after the prompt, and whether it is in the history."""
    offsets = s["offsets"]
    lo, hi = s["edges"][first], s["edges"][last]
    rows, at = _plain_rows_of(offsets, lo, hi, first, last)
    flat = rows * V + s["tokens"][lo:hi]
    made = (at - offsets[first:last][rows] >= s["n_prompt"][first:last][rows]).float()
    count = torch.zeros((last - first) * V, device=DEV)
    seen = torch.zeros((last - first) * V, dtype=torch.bool, device=DEV)
    count.scatter_add_(0, flat, made)
    seen[flat] = True
    return count.view(-1, V), seen.view(-1, V)


def _plain_allowed(s, first, last, V):
    if s["allowed"] is None:
        return None
    mask = s["mask"][first:last]
    words = s["allowed"][mask.clamp(min=0)]
    bits = (words[:, :, None] >> torch.arange(32, device=DEV, dtype=torch.int32)) & 1
    return (bits.reshape(last - first, -1)[:, :V] != 0) | (mask < 0)[:, None]


def _plain_adjust(s, grad):
    x, parts = s["x"], []
    T, V = x.shape
    step = max(1, (1 << 27) // V)
    for first in range(0, T, step):
        last = min(first + step, T)
        part = slice(first, last)
        v = x[part].float()
        count, seen = _plain_seen(s, first, last, V)
        rep = s["repetition"][part, None]
        ok = _plain_allowed(s, first, last, V)
        if grad:
            d = s["dy"][part].float()
            d = torch.where(seen, torch.where(v > 0, d / rep, d * rep), d)
            if ok is not None:
                d = torch.where(ok, d, torch.zeros_like(d))
            parts.append(d.to(x.dtype))
            continue
        u = torch.where(seen, torch.where(v > 0, v / rep, v * rep), v)
        u = u - (count > 0).float() * s["presence"][part, None] - count * s["frequency"][part, None]
        if s["bias"] is not None:
            ids, values, offsets = s["bias"]
            lo, hi = first * s["case"]["biases"], last * s["case"]["biases"]
            rows, _ = _plain_rows_of(offsets, lo, hi, first, last)
            u.view(-1).scatter_add_(0, rows * V + ids[lo:hi], values[lo:hi])
        if ok is not None:
            u = u.masked_fill(~ok, -math.inf)
        parts.append(u.to(x.dtype))
    return torch.cat(parts) if len(parts) > 1 else parts[0]


def run(s):
    kind, case = s["kind"], s["case"]
    if own:
        import paper_2608_12573_amd as pk
        if kind == "norm":
            return pk.layer_norm(s["x"], s["w"], s["b"], eps=EPS, out=s["out"])
        if kind == "norm_grad":
            return pk.layer_norm_grad(s["dy"], s["x"], s["w"], s["mean"], s["rstd"], ws=s["ws"], out=s["out"])
        if kind == "linear":
            return pk.linear(s["x"], s["w"], s["b"], activation=case["act"], residual=s["r"], ws=s["ws"], out=s["out"])
        if kind == "linear_grad":
            return pk.linear_grad(s["r"], s["x"], s["w"], s["z"], activation=case["act"], ws=s["ws"], out=s["out"])
        rows = dict(n_prompt=s["n_prompt"], repetition=s["repetition"], allowed=s["allowed"], mask=s["mask"],
                    out=s["out"])
        if kind == "adjust":
            return pk.adjust_logits(s["x"], s["tokens"], s["offsets"], presence=s["presence"],
                                    frequency=s["frequency"], bias=s["bias"], **rows)
        return pk.adjust_logits_grad(s["dy"], s["x"], s["tokens"], s["offsets"], **rows)
    if kind == "norm":
        return _plain_norm(s["x"], s["w"], s["b"], DTYPE[case["out"]])
    if kind == "norm_grad":
        return _plain_norm_grad(s)
    if kind == "linear":
        return _plain_linear(s)
    if kind == "linear_grad":
        return _plain_linear_grad(s)
    return _plain_adjust(s, kind == "adjust_grad")


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        n, T, D = case["T"] * case["D"], case["T"], case["D"]
        i, o = BYTES[case["dtype"]], BYTES[case["out"]]
        if kind == "norm":           # rows, scale and shift in; rows and statistics out
            return {"bytes": n * (i + o) + 8 * D + 8 * T, "flops": 8 * n}
        # the gradient, rows, scale and statistics in; three gradients out
        return {"bytes": n * (2 * i + o) + 12 * D + 8 * T, "flops": 14 * n}
    if kind in ("linear", "linear_grad"):
        M, K, N = case["M"], case["K"], case["N"]
        o = BYTES[case["out"]]
        if kind == "linear":
            return {"bytes": 2 * (M + N) * K + M * N * o * (2 if case["residual"] else 1) + 4 * N * bool(case["bias"]),
                    "flops": 2 * M * N * K}
        # (without an activation the kept z need not be read)
        return {"bytes": 4 * (M + N) * K + M * N * o * (2 if case["act"] else 1) + 4 * N, "flops": 4 * M * N * K}
    n, T = case["T"] * case["V"], case["T"]
    # logits in and out, or the gradient in and out and the logits of the
    # tokens that were seen; three quarters of the longest history, its lists
    # and the masks' bits once each
    history = T * case["history"] * 3 // 4
    lists = 8 * history + 12 * T * case["biases"] + 40 * T + case["masks"] * (case["V"] // 8)
    gather = history * BYTES[case["dtype"]] if kind == "adjust_grad" else 0
    return {"bytes": 2 * n * BYTES[case["dtype"]] + lists + gather, "flops": 4 * n}


# ------------------------------------------------------------- in 64 bits ---

def _exact_norm(case, seed):
    x, w, b, dy = _norm_inputs(case, seed)
    T = case["T"]
    step = max(1, (1 << 26) // case["D"])
    y, means, scales = [], [], []
    for r in range(0, T, step):
        z = x[r:r + step].double()
        var, m = torch.var_mean(z, dim=1, keepdim=True, unbiased=False)
        scale = torch.rsqrt(var + EPS)
        y.append(torch.addcmul(b.double(), (z - m) * scale, w.double()))
        means.append(m[:, 0])
        scales.append(scale[:, 0])
    return torch.cat(y), torch.cat(means), torch.cat(scales)


def _exact_norm_grad(case, seed):
    """With the statistics that the call is given."""
    x, w, b, dy = _norm_inputs(case, seed)
    _, mean, rstd = _plain_norm(x, w, b, torch.float32)
    T, D = case["T"], case["D"]
    dx = torch.empty((T, D), dtype=torch.float64, device=DEV)
    dw = torch.zeros(D, dtype=torch.float64, device=DEV)
    db = torch.zeros(D, dtype=torch.float64, device=DEV)
    step = max(1, (1 << 26) // D)
    for r in range(0, T, step):
        scale = rstd[r:r + step, None].double()
        n = x[r:r + step].double().sub_(mean[r:r + step, None].double()).mul_(scale)
        u = dy[r:r + step].double()
        dw += torch.mul(n, u).sum(dim=0)
        db += u.sum(dim=0)
        u *= w.double()
        # the part of the gradient along 1 and along n is taken out
        along = torch.bmm(u[:, None], n[:, :, None].contiguous())[:, 0] / D
        dx[r:r + step] = (u - u.sum(dim=1, keepdim=True) / D - n * along) * scale
    return dx, dw, db


def _exact_act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, 0.0)
    if act == "gelu":
        return z * torch.special.ndtr(z)
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _exact_slope(z, act):
    if act == "relu":
        return torch.where(z > 0, 1.0, 0.0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        p = torch.sigmoid(z)
        return p + z * p * torch.sigmoid(-z)
    return torch.ones_like(z)


def _exact_linear(case, seed):
    x, w, b, r = _linear_inputs(case, seed)
    out = torch.empty((case["M"], case["N"]), dtype=torch.float64, device=DEV)
    a = x.double()
    for c in range(0, case["N"], 8192):
        z = torch.mm(a, w[c:c + 8192].double().t())
        if b is not None:
            z += b[c:c + 8192].double()
        z = _exact_act(z, case["act"])
        out[:, c:c + 8192] = z if r is None else z + r[:, c:c + 8192].double()
    return out


def _exact_linear_grad(case, seed):
    x, w, b, dy = _linear_inputs(case, seed)
    z = _plain_product(x, w, b).to(DTYPE[case["out"]])
    dz = _exact_slope(z.double(), case["act"]).mul_(dy.double())
    return torch.mm(dz, w.double()), torch.mm(x.double().t(), dz).t(), dz.sum(dim=0)


def _exact_adjust(case, seed):
    """Row by row, each token of the history at its place."""
    s = _adjust_inputs(case, seed)
    grad = case["kind"] == "adjust_grad"
    T, V = case["T"], case["V"]
    out = (s["dy"] if grad else s["x"]).double()
    offsets, prompts = s["offsets"].tolist(), s["n_prompt"].tolist()
    masks = s["mask"].tolist() if case["masks"] else [-1] * T
    bits = None
    if case["masks"]:
        shift = torch.arange(32, device=DEV)
        bits = [((m.to(torch.int64)[:, None] >> shift) % 2 == 1).view(-1)[:V] for m in s["allowed"]]
    rep = s["repetition"].double()
    for r in range(T):
        ids = torch.unique(s["tokens"][offsets[r]:offsets[r + 1]])
        x = s["x"][r, ids].double()
        up = x > 0
        if grad:
            out[r, ids] *= torch.where(up, 1.0 / rep[r], rep[r])
        else:
            made = torch.bincount(s["tokens"][offsets[r] + prompts[r]:offsets[r + 1]], minlength=V)[ids].double()
            x = torch.where(up, x / rep[r], x * rep[r])
            out[r, ids] = x - (made >= 1) * s["presence"][r].double() - made * s["frequency"][r].double()
            if s["bias"] is not None:
                k = case["biases"]
                out[r, s["bias"][0][r * k:(r + 1) * k]] += s["bias"][1][r * k:(r + 1) * k].double()
        if masks[r] >= 0:
            out[r].masked_fill_(~bits[masks[r]], 0.0 if grad else -math.inf)
    return out


def exact(case, seed):
    return dict(norm=_exact_norm, norm_grad=_exact_norm_grad, linear=_exact_linear, linear_grad=_exact_linear_grad,
                adjust=_exact_adjust, adjust_grad=_exact_adjust)[case["kind"]](case, seed)
