"""Attention layers in 64 bits, from the definitions (test infrastructure; shares no code with the library).

numpy only, one sequence and head at a time.  The bounds that come with the results say how far a correct 16-bit kernel may be off, entry by entry: every
rounding to bfloat16 is at most ROUND = 2^-8 of the rounded value (half an ulp of its 8 bits), SLACK covers the 32-bit sums and exponentials around it.
"""
from __future__ import annotations

import numpy as np

ROUND = 2.0 ** -8
SLACK = 2e-5
GROUP = 64


def looked_at(nq: int, nk: int, causal: bool) -> np.ndarray:
    """Which keys (columns) each query (row) looks at; causal: the last query at all of them."""
    if not causal:
        return np.ones((nq, nk), dtype=bool)
    return np.arange(nk)[None, :] - (nk - nq) <= np.arange(nq)[:, None]


def attention(q, k, v, scale, causal):
    """(out, lse, weights, bound of out) of one head: q (nq, d), k, v (nk, d) float64."""
    nq, nk = len(q), len(k)
    seen = looked_at(nq, nk, causal)
    out, lse, p = np.zeros(q.shape), np.full(nq, -np.inf), np.zeros((nq, nk))
    size = np.zeros(q.shape)
    for i in range(nq):
        j = np.flatnonzero(seen[i])
        if len(j) == 0:
            continue
        s = scale * (k[j] @ q[i])
        top = s.max()
        e = np.exp(s - top)
        lse[i] = top + np.log(e.sum())
        p[i, j] = e / e.sum()
        out[i] = p[i, j] @ v[j]
        size[i] = p[i, j] @ np.abs(v[j])
    # weights rounded, the result rounded
    return out, lse, p, 1.02 * ROUND * (size + np.abs(out)) + SLACK * size + 1e-30


def attention_backward(q, k, v, scale, causal, dout):
    """((dq, dk, dv), their bounds) of one head."""
    out, _, p, out_bound = attention(q, k, v, scale, causal)
    dp = dout @ v.T
    delta = (dout * out).sum(1, keepdims=True)
    ds = p * (dp - delta)
    dq, dk, dv = scale * ds @ k, scale * ds.T @ q, p.T @ dout
    # dS: its own rounding, and that of out in delta; P in dv is rounded
    spread = p * (np.abs(dout) * out_bound).sum(1, keepdims=True)
    off = ROUND * np.abs(ds) + spread + SLACK * p * (np.abs(dout) @ np.abs(v).T + np.abs(dout * out).sum(1, keepdims=True))
    bq = scale * off @ np.abs(k) + ROUND * np.abs(dq)
    bk = scale * off.T @ np.abs(q) + ROUND * np.abs(dk)
    bv = (ROUND + SLACK) * p.T @ np.abs(dout) + ROUND * np.abs(dv)
    return (dq, dk, dv), tuple(1.02 * b + 1e-30 for b in (bq, bk, bv))


def turn(y, cos, sin, interleaved, back=False):
    """y (heads, d) of one token turned by its angles, cos and sin (r / 2,)."""
    z = y.copy()
    h = len(cos)
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        s = -sin[i] if back else sin[i]
        z[:, a] = y[:, a] * cos[i] - y[:, b] * s
        z[:, b] = y[:, b] * cos[i] + y[:, a] * s
    return z


def norm_rope(x, weight, cos, sin, interleaved, eps):
    """x (heads, d) of one token."""
    r = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    return turn(x * r * weight, cos, sin, interleaved)


def norm_rope_backward(dz, x, weight, cos, sin, interleaved, eps):
    """(dx, dweight) of one token."""
    r = 1.0 / np.sqrt((x * x).mean(1, keepdims=True) + eps)
    u = x * r
    dy = turn(dz, cos, sin, interleaved, back=True)
    du = dy * weight
    return r * (du - u * (du * u).mean(1, keepdims=True)), (dy * u).sum(0)


def to_bf16(x):
    """float64 or float32 to the nearest bfloat16 (ties to even), as float32; for finite values and NaN."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7fff + ((b >> 16) & 1)) & 0xffff0000).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(np.asarray(x, dtype=np.float32)), np.float32(np.nan), r)


def quantise(x):
    """(step, low, n) of one group of 64 float32 values."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(over="ignore", invalid="ignore"):
        span = np.float32(x.max()) - np.float32(x.min())
    if not np.isfinite(x).all() or not np.isfinite(span):
        return np.float32(np.nan), np.float32(np.nan), np.zeros(GROUP, dtype=np.int64)
    step, low = np.float32(to_bf16(np.float32(span / np.float32(15)))), np.float32(x.min())
    if step == 0:
        return step, low, np.zeros(GROUP, dtype=np.int64)
    return step, low, np.minimum(np.rint((x - low) / step), 15).astype(np.int64)


def word(numbers) -> int:
    """Eight numbers of 0..15 as the cache packs them: number 2 i + h in bits 4 (i + 4 h)."""
    w = 0
    for i in range(4):
        for h in range(2):
            w |= int(numbers[2 * i + h]) << (4 * (i + 4 * h))
    return w


def decode(q, k, v, step, n, scale):
    """(out, bound) of one query over a head's cached keys and values (float64), v = low + step n given with its step and numbers (tokens, d):
    the weights times step are rounded, against n - 8."""
    if len(k) == 0:
        return np.zeros(len(q)), np.full(len(q), 1e-30)
    s = scale * (k @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    out = p @ v
    return out, 1.02 * ROUND * (p @ np.abs(step * (n - 8)) + np.abs(out)) + SLACK * (p @ (np.abs(v) + 136 * step)) + 1e-30
