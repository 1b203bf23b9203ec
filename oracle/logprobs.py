"""O4: log probabilities of tokens, entropy and alternatives of rows of
logits, and their gradient, in fp64.

Test infrastructure (see the package docstring).  Rows are fp64 arrays that
hold fp32 or bf16 values exactly.  With p = exp(x - lse), lse = log sum exp(x):
    logprob = x_y - lse,   H = -sum p log p (0 log 0 = 0),
    alternatives = the n largest x, ties by smaller index.
Cases without a value of their own: a negative token has logprob 0, a token
past the row NaN; -inf logits have p = 0 and are never alternatives; a row of
nothing else has lse = logprob = -inf and H = 0; NaN or +inf make the row's
statistics NaN.
"""

import numpy as np


# From this size on fp32 holds an lse too coarsely for p = exp(x - lse).
COARSE_LSE = 16384.0


def log_softmax(x):
    """x - m, then less the logarithm of the sum: m + log s would lose the
    latter beside an m of the lowest value."""
    m = x.max()
    with np.errstate(all="ignore"):
        return (x - m) - np.log(np.exp(x - m).sum())


def row(x, y, n):
    """(logprob, H, lse, alternatives' log probabilities, their indices) of
    one row; the alternatives are padded with (-inf, -1)."""
    x = np.asarray(x, dtype=np.float64)
    V = x.size
    with np.errstate(all="ignore"):
        l = np.full(V, -np.inf)
        if np.any(np.isnan(x)) or np.any(x == np.inf):
            lse = h = np.nan
            l[:] = np.nan
        elif np.all(x == -np.inf):
            lse, h = -np.inf, 0.0
        else:
            l = log_softmax(x)
            m = x.max()
            lse = m + np.log(np.exp(x - m).sum())
            p = np.exp(l)
            h = -np.sum(p[p > 0] * l[p > 0])
        if y < 0:
            lp = 0.0
        else:
            lp = np.nan if y >= V else l[y]
        # total order: by bit pattern, so -0 lies below +0 and +NaN on top
        b = x.view(np.int64)
        key = np.where(b < 0, -(b & 0x7FFFFFFFFFFFFFFF) - 1, b)
        floor = np.float64(-np.inf).view(np.int64)
        floor = -(int(floor) & 0x7FFFFFFFFFFFFFFF) - 1
        idx = np.argsort(-key.astype(object), kind="stable") if V < 64 else np.lexsort((np.arange(V), ~key))
        idx = np.array([i for i in idx[:n] if key[i] > floor], dtype=np.int64)
        top = np.full(n, -np.inf)
        top[:idx.size] = l[idx]
        out = np.full(n, -1, dtype=np.int64)
        out[:idx.size] = idx
    return lp, h, lse, top, out


def rows(x, y, n):
    """row() of every row, stacked."""
    res = [row(x[r], int(y[r]), n) for r in range(len(y))]
    return tuple(np.array([q[i] for q in res]) for i in range(3)) + \
        tuple(np.stack([q[i] for q in res]) if res else np.zeros((0, n)) for i in (3, 4))


def grad_row(x, y, lse, h, g_lp, g_h, top_idx, g_top):
    """Gradient of g_lp logprob + g_h H + sum g_top (x[top_idx] - lse) with
    respect to x, with p = exp(x - lse) from the given lse and H (from x itself
    where an fp32 lse is too coarse)."""
    x = np.asarray(x, dtype=np.float64)
    V = x.size
    d = np.zeros(V)
    if lse == -np.inf:
        return d
    if np.isnan(lse) or (y >= V and g_lp is not None):
        return np.full(V, np.nan)
    l = x - lse if abs(lse) < COARSE_LSE else log_softmax(x)
    p = np.exp(l)
    total = 0.0
    if g_lp is not None and y >= 0:
        total += g_lp
        d[y] += g_lp
    for j, t in zip(top_idx, g_top):
        if 0 <= j < V:
            total += t
            d[j] += t
    on = p > 0
    d[on] -= p[on] * total
    if g_h is not None:
        d[on] -= g_h * p[on] * (l[on] + h)
    return d


def grad_of_logits(x, y, g_lp, g_h, top_idx, g_top, g_lse=0.0):
    """The gradient of grad_row's sum and g_lse lse, from the logits alone: the
    gradients of the log probabilities l, then through l = x - lse
    (dl_i/dx_j = [i = j] - p_j); H = -sum p l adds -p (l + 1) to the former, and
    lse has the gradient p.  A row with a value of its own (finite lse), y below
    V."""
    x = np.asarray(x, dtype=np.float64)
    l = log_softmax(x)
    p = np.exp(l)
    u = np.zeros(x.size)
    if g_lp is not None and y >= 0:
        u[y] += g_lp
    for j, t in zip(top_idx, g_top):
        if 0 <= j < x.size:
            u[j] += t
    if g_h is not None:
        on = p > 0
        u[on] -= g_h * p[on] * (l[on] + 1.0)
    return u + p * (g_lse - u.sum())


def grad_scale(x, y, lse, h, g_lp, g_h, top_idx, g_top):
    """The magnitude that a rounded gradient's error is proportional to: the
    sum of the terms' magnitudes, each p's error growing with |x - lse|."""
    x = np.asarray(x, dtype=np.float64)
    V = x.size
    if not np.isfinite(lse):
        return np.zeros(V)
    l = np.maximum(x - lse if abs(lse) < COARSE_LSE else log_softmax(x), -1e4)
    p = np.exp(l)
    total = (abs(g_lp) if g_lp is not None and 0 <= y < V else 0.0) + np.abs(g_top).sum()
    s = p * (total + (abs(g_h) * (np.abs(l) + abs(h)) if g_h is not None else 0.0)) * (8.0 + 2.0 * np.abs(l))
    if g_lp is not None and 0 <= y < V:
        s[y] += abs(g_lp) * (2 + len(g_top))
    for j, t in zip(top_idx, g_top):
        if 0 <= j < V:
            s[j] += abs(t) * (2 + len(g_top))
    return s
