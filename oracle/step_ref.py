"""What a group rollout's decode step does around and in its attention, written plainly in 64 bits.

TEST INFRASTRUCTURE ONLY. Rotary positions, attention of sequences that share their
first pages, and sampling; one token, row and entry after the other.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def frequencies(turn, base, factor=None, trained=0.0, low=1.0, high=4.0):
    out = []
    for i in range(turn // 2):
        f = base ** (-2.0 * i / turn)
        if factor is not None:
            stay = 0.0
            if trained > 0:
                stay = min(1.0, max(0.0, (trained * f / (2 * math.pi) - low) / (high - low)))
            f = stay * f + (1 - stay) * f / factor
        out.append(f)
    return np.array(out)


def rotate(x, position, freq, interleaved, magnitude=1.0):
    """Head vectors x [H, D] (float64) at one position; and the sizes of what each result is the difference of."""
    y, size = x.copy(), np.abs(x)
    half = freq.size
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, half + i)
        c, s = math.cos(position * f) * magnitude, math.sin(position * f) * magnitude
        y[:, a], y[:, b] = x[:, a] * c - x[:, b] * s, x[:, b] * c + x[:, a] * s
        size[:, a] = size[:, b] = (np.abs(x[:, a]) + np.abs(x[:, b])) * abs(magnitude)
    return y, size


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def attend(q, k, v, scale):
    """Rows q [R, D] over keys k and values v [L, D]: (out, lse, sum of p |v|, largest sum of |q k| scale)."""
    if k.shape[0] == 0:
        return np.zeros_like(q), np.full(q.shape[0], -np.inf), np.zeros_like(q), np.zeros(q.shape[0])
    z = (q @ k.T) * scale
    top = z.max(1, keepdims=True)
    p = np.exp(z - top)
    total = p.sum(1, keepdims=True)
    p /= total
    size = (np.abs(q) @ np.abs(k).T * abs(scale)).max(1)
    return p @ v, (top + np.log(total))[:, 0], p @ np.abs(v), size


# ---------------------------------------------------------------------------
# sampling
# ---------------------------------------------------------------------------
def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row (float64). Returns ({token: logprob}, kept): the token, and those among what stays to whose
    share of the sum the draw is nearer than V 2^-43 of everything."""
    x = np.where(np.isnan(logits), -np.inf, logits)
    n = x.size
    top = x.max()
    if top == -np.inf:
        return {-1: -np.inf}, 0.0
    greedy = not temperature > 0
    t = 1.0 if greedy else temperature
    if top == np.inf:
        y = np.where(x == np.inf, 0.0, -np.inf)
    else:
        with np.errstate(invalid="ignore", over="ignore"):
            y = np.where(x == -np.inf, -np.inf, (x - top) / t)
    w = np.exp(y)
    total = math.fsum(w)
    if greedy:
        at = int(np.argmax(x))
        return {at: y[at] - math.log(total)}, w[at] / total
    order = sorted(range(n), key=lambda v: (-x[v], v))
    if 0 < top_k < n:
        order = order[:top_k]
    if top_p < 1:   # (False for NaN)
        whole, before, stay = math.fsum(w[order]), 0.0, []
        for v in order:
            if stay and not before < top_p * whole:
                break
            stay.append(v)
            before += w[v]
        order = stay
    if min_p > 0:
        order = [v for v in order if w[v] >= min(min_p, 1.0)]
    keep = sorted(order)
    whole = math.fsum(w[keep])
    u = min(u, 1 - 2.0 ** -24) if u > 0 else 0.0
    cum, off = np.cumsum(w[keep]), n * 2.0 ** -43 * total
    near = (cum - w[keep] <= u * whole + off) & (cum >= u * whole - off)
    return {keep[i]: y[keep[i]] - math.log(total) for i in np.flatnonzero(near)}, whole / total
