"""Layer norm, dense product and adjusted logits with their gradients in fp64
(numpy), from their formulas."""

import numpy as np
from scipy.special import erf, expit


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """(y, mean, rstd) of the rows of x."""
    x = np.asarray(x, np.float64)
    m = x.mean(axis=1)
    c = x - m[:, None]
    with np.errstate(divide="ignore", invalid="ignore"):
        r = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
        y = c * r[:, None]
    if weight is not None:
        y = y * weight
    if bias is not None:
        y = y + bias
    return y, m, r


def layer_norm_grad(dy, x, weight, mean, rstd):
    """(dx, dweight, dbias) with the given statistics."""
    dy, x = np.asarray(dy, np.float64), np.asarray(x, np.float64)
    r = np.asarray(rstd, np.float64)[:, None]
    n = (x - np.asarray(mean, np.float64)[:, None]) * r
    g = dy if weight is None else dy * weight
    dx = r * (g - g.mean(axis=1, keepdims=True) - n * (g * n).mean(axis=1, keepdims=True))
    return dx, (dy * n).sum(axis=0), dy.sum(axis=0)


def act(z, name):
    if name == "relu":
        return np.where(z < 0, 0.0, z)
    if name == "gelu":
        return np.where(np.isneginf(z), 0.0, 0.5 * z * (1.0 + erf(z / np.sqrt(2.0))))
    if name == "silu":
        return np.where(np.isneginf(z), 0.0, z * expit(z))
    return z


def slope(z, name):
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if name == "gelu":
        c = np.clip(z, -100, 100)
        return 0.5 * (1.0 + erf(c / np.sqrt(2.0))) + c * np.exp(-0.5 * c * c) / np.sqrt(2.0 * np.pi)
    if name == "silu":
        c = np.clip(z, -500, 500)
        p = expit(c)
        return p * (1.0 + c * (1.0 - p))
    return np.ones_like(z)


def linear(x, w, bias=None, activation=None, residual=None):
    """(y, z)."""
    z = np.asarray(x, np.float64) @ np.asarray(w, np.float64).T
    if bias is not None:
        z = z + bias
    y = act(z, activation)
    return (y if residual is None else y + residual), z


def linear_grad(dy, x, w, z, activation=None):
    """(dx, dw, db, dz)."""
    dz = np.asarray(dy, np.float64)
    if activation is not None:
        dz = dz * slope(np.asarray(z, np.float64), activation)
    return dz @ np.asarray(w, np.float64), dz.T @ np.asarray(x, np.float64), dz.sum(axis=0), dz


def _row(r, V, tokens, offsets, n_prompt):
    """Occurrences after the prompt, and whether a token is in the history."""
    made, seen = np.zeros(V), np.zeros(V, bool)
    if tokens is None:
        return made, seen
    lo = min(max(int(offsets[r]), 0), len(tokens))
    hi = min(max(int(offsets[r + 1]), lo), len(tokens))
    prompt = 0 if n_prompt is None else min(max(int(n_prompt[r]), 0), hi - lo)
    for k, t in enumerate(tokens[lo:hi]):
        if 0 <= t < V:
            seen[t] = True
            made[t] += k >= prompt
    return made, seen


def _mask(r, T, V, allowed, mask):
    """Which tokens row r may take (None: it names a mask that is not there)."""
    if allowed is None:
        return np.ones(V, bool)
    k = int(mask[r]) if mask is not None else 0 if len(allowed) == 1 else r
    if k < 0:
        return np.ones(V, bool)
    if k >= len(allowed):
        return None
    word = np.asarray(allowed[k]).astype(np.int64) & 0xFFFFFFFF
    v = np.arange(V)
    return (word[v // 32] >> (v % 32)) & 1 == 1


def adjust(x, tokens=None, offsets=None, n_prompt=None, repetition=None, presence=None, frequency=None, bias=None,
           allowed=None, mask=None):
    x = np.array(x, np.float64)
    T, V = x.shape
    for r in range(T):
        made, seen = _row(r, V, tokens, offsets, n_prompt)
        rep = 1.0 if repetition is None else float(repetition[r])
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            y = np.where(seen, np.where(x[r] > 0, x[r] / rep, x[r] * rep), x[r])
        if presence is not None:
            y = y - (made > 0) * float(presence[r])
        if frequency is not None:
            y = y - made * float(frequency[r])
        if bias is not None:
            ids, values, at = bias
            lo = min(max(int(at[r]), 0), len(ids))
            last = {int(t): float(v) for t, v in zip(ids[lo:max(int(at[r + 1]), lo)], values[lo:max(int(at[r + 1]), lo)])}
            for t, v in last.items():
                if 0 <= t < V:
                    y[t] += v
        ok = _mask(r, T, V, allowed, mask)
        x[r] = np.nan if ok is None else np.where(ok, y, -np.inf)
    return x


def adjust_grad(d, x, tokens=None, offsets=None, repetition=None, allowed=None, mask=None):
    d, x = np.array(d, np.float64), np.asarray(x, np.float64)
    T, V = x.shape
    for r in range(T):
        _, seen = _row(r, V, tokens, offsets, None)
        rep = 1.0 if repetition is None else float(repetition[r])
        f = np.where(seen, np.where(x[r] > 0, 1.0 / rep, rep), 1.0)
        ok = _mask(r, T, V, allowed, mask)
        d[r] = np.nan if ok is None else np.where(ok, d[r] * f, 0.0)
    return d
