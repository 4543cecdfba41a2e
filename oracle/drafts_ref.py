"""A step with drafted tokens in 64 bits, from the definitions (test infrastructure; shares no code with the library).

numpy only, one sequence at a time.  Bounds as in attention_ref.py: how far a correct 16-bit kernel may be off, entry by entry.
"""
from __future__ import annotations

import numpy as np

from oracle.attention_ref import ROUND, SLACK, turn


def turned(x, cos, sin, interleaved):
    """(z, bound): x (heads, d) of one token turned by its angles; the result is rounded once, its two products and their sum to 24 bits."""
    z = turn(x, cos, sin, interleaved)
    size = np.abs(turn(np.abs(x), np.abs(cos), -np.abs(sin), interleaved)) + np.abs(turn(np.abs(x), np.abs(cos), np.abs(sin), interleaved))
    return z, 1.01 * ROUND * np.abs(z) + 2.0 ** -22 * size + 1e-38


def looked_at(n: int, length: int, masks=None) -> np.ndarray:
    """Which of `length` positions, the last n of which are a block's tokens, each token looks at; masks: bit j for token j of the block, None: up to itself."""
    seen = np.zeros((n, length), dtype=bool)
    for i in range(n):
        for at in range(length):
            j = at - (length - n)
            seen[i, at] = j < 0 or (j <= i if masks is None else j < 64 and bool(masks[i] >> j & 1))
    return seen


def attention(q, k, v, scale, seen):
    """(out, bound) of one head: q (n, d), k, v (length, d) float64, seen (n, length)."""
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    rows = seen.any(1)
    if rows.any():
        s = np.where(seen[rows], scale * (q[rows] @ k.T), -np.inf)
        e = np.exp(s - s.max(1, keepdims=True))
        e /= e.sum(1, keepdims=True)
        out[rows], size[rows] = e @ v, e @ np.abs(v)
    return out, 1.02 * ROUND * (size + np.abs(out)) + SLACK * size + 1e-30


def verify(target, tokens, uniforms, draft=None, parents=None):
    """(accepted, path, token) of one block: target (n, vocab) and draft float64, the rest lists of numbers; path has n entries."""
    n, vocab = target.shape
    if n == 0:
        return 0, [], -1
    target = np.where(target < 0, 0.0, target)
    draft = None if draft is None else np.where(draft < 0, 0.0, draft)
    parents = [i - 1 for i in range(n)] if parents is None else parents
    path, tested = [0], 0
    p, mass = target[0].copy(), 1.0
    while True:
        node = path[-1]
        c = next((i for i in range(tested + 1, min(n, 64)) if parents[i] == node and 0 <= node < i and 0 <= tokens[i] < vocab), None)
        if c is None:
            break
        tested, x, u = c, tokens[c], float(uniforms[c])
        with np.errstate(invalid="ignore"):
            if u * draft[node, x] < p[x] if draft is not None else p[x] > max(u * mass, 0.0):
                path.append(c)
                p, mass = target[c].copy(), 1.0
            elif draft is None:
                mass -= p[x]
                p[x] = 0.0
            else:
                rest = p - draft[node]
                rest = np.where(rest < 0, 0.0, rest)
                total = rest.sum()
                p = rest / total if total > 0 else p
    total = p.sum()
    token = -1
    if total > 0 and np.isfinite(total):
        over = np.flatnonzero(np.cumsum(p) > float(uniforms[0]) * total)
        token = int(over[0]) if len(over) else int(np.flatnonzero(p > 0)[-1])
    return len(path) - 1, path + [-1] * (n - len(path)), token
