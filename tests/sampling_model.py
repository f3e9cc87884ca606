"""What rotary positions, attention over a shared prefix and sampling are to compute, in numpy and 64
bits, written from their definitions."""

import math

import numpy as np

U24 = 2.0 ** -24
ONE = 2.0 ** 43   # what a weight of 1 counts in sampling


# ---- rotary positions ----

def freqs(dims, base, factor=1.0, original=0.0, low=0.0, high=0.0, ramp=0):
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        if ramp == 0:
            r = 0.0
        elif ramp == 1:
            r = (original * f / (2 * math.pi) - low) / (high - low)
        else:
            c = [dims * math.log(original / (2 * math.pi * n)) / (2 * math.log(base)) for n in (high, low)]
            a, b = max(0, math.floor(c[0])), min(dims - 1, math.ceil(c[1]))
            r = 1 - (i - a) / ((b - a) or 0.001)
        r = min(1.0, max(0.0, r))
        out.append(f * (r + (1 - r) / factor))
    return out


def rotate(x, pos, freq, interleaved, factor, norm, eps):
    """x [tokens, heads, dim] -> (y, bound on what fp32 may be off by before the output's rounding)."""
    x = np.asarray(x, np.float64)
    n, _, dim = x.shape
    size = np.abs(x)
    # a mean of `dim` squares in fp32 errs by (dim + 2) 2^-24 of itself, its root by half, and four roundings more
    err = np.zeros(1)
    if norm is not None:
        x = x / np.sqrt((x * x).mean(2, keepdims=True) + eps) * norm
        size = np.abs(x)
        err = size * ((dim + 2) / 2 + 6) * U24
    y, bound = x.copy(), err + np.zeros_like(x)
    half = len(freq)
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(pos, np.float64) * f
        # fp64 holds the angle to 2^-53 of itself in each of four steps here and there; cosine and sine in
        # fp32 are good to 4 units in the last place (2^-23 each), and three products and a sum follow
        off = np.abs(t) * 2.0 ** -50 + 4 * 2.0 ** -23 + 4 * U24
        c, s = np.cos(t)[:, None], np.sin(t)[:, None]
        y[:, :, a], y[:, :, b] = factor * (x[:, :, a] * c - x[:, :, b] * s), factor * (x[:, :, b] * c + x[:, :, a] * s)
        both = size[:, :, a] + size[:, :, b]
        worst = factor * (both * off[:, None] + (0 if norm is None else err[:, :, a] + err[:, :, b]))
        bound[:, :, a] = bound[:, :, b] = worst
    return y, bound


# ---- attention ----

def attention(q, k, v, scale):
    """Queries [heads, dim] of one key head over its tokens k, v [tokens, dim]: (y, lse, sum of p |v|, largest
    sum of |q k| times scale)."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    if len(k) == 0:
        return np.zeros(q.shape), np.full(len(q), -np.inf), np.zeros(q.shape), np.zeros(len(q))
    s = q @ k.T * scale
    top = s.max(1, keepdims=True)
    e = np.exp(s - top)
    w = e / e.sum(1, keepdims=True)
    return w @ v, top[:, 0] + np.log(e.sum(1)), w @ np.abs(v), (np.abs(q) @ np.abs(k).T).max(1) * abs(scale)


# ---- sampling ----

def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (token, log probability, its weight)."""
    l = np.asarray(logits, np.float64)
    order = np.argsort(-np.where(np.isnan(l), -np.inf, l), kind="stable")
    order = order[l[order] > -np.inf]
    if len(order) == 0:
        return -1, -np.inf, 0.0
    top = l[order[0]]
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    with np.errstate(invalid="ignore"):
        w = np.where(l[order] == top, 1.0, 0.0 if top == np.inf else np.exp((l[order] - top) / temperature))
    m = np.rint(w * ONE).astype(np.uint64)
    n = len(order)
    if top_k > 0:
        n = min(n, top_k)
    if top_p < 1:
        need = max(1, math.ceil(max(float(top_p), 0.0) * float(int(m[:n].sum()))))
        n = min(n, int(np.searchsorted(np.cumsum(m[:n]), np.uint64(need))) + 1)
    if min_p > 0:
        n = max(1, min(n, int(((w >= min_p) | (l[order] == top)).sum())))
    kept = np.sort(order[:n])
    m = np.rint(np.where(l[kept] == top, 1.0, 0.0 if top == np.inf else np.exp((l[kept] - top) / temperature)) * ONE).astype(np.uint64)
    total = int(m.sum())
    u = min(max(float(u), 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    i = int(np.searchsorted(np.cumsum(m), np.uint64(int(u * float(total))), side="right"))
    return int(kept[i]), math.log(int(m[i]) / total), int(m[i]) / ONE
