"""fp64 oracle of the adjustment of logits and of the token history."""
from __future__ import annotations

import numpy as np

MOST = 16383


def path(parents, row):
    """Nodes on the way to a row, itself included, the root excluded (parents None: a chain)."""
    nodes = []
    while row > 0:
        nodes.append(row)
        p = row - 1 if parents is None else int(parents[row - 1])
        row = p if 0 <= p < row else 0
    return nodes


def adjust_row(x, history=None, drafted=(), r=1.0, p=0.0, f=0.0, bias=(), allowed=None):
    """One row: `drafted` are the tokens on its way, `bias` pairs (token, value), `allowed` truth values."""
    x = np.asarray(x, np.float64).copy()
    V = len(x)
    count = np.zeros(V) if history is None else (np.asarray(history) // 2).astype(np.float64)
    seen = np.zeros(V, bool) if history is None else np.asarray(history) != 0
    for t in drafted:
        if 0 <= t < V:
            count[t] += 1
            seen[t] = True
    x = np.where(seen, np.where(x > 0, x / r, x * r), x)
    x = np.where(count > 0, x - f * count - p, x)
    for t, b in bias:
        if 0 <= t < V:
            x[t] += b
    if allowed is not None:
        x = np.where(allowed, x, -np.inf)
    return x


def enter(history, fresh=None, prompts=None, emitted=None):
    """history [B, V] after the call: prompts and emitted are lists of token lists."""
    h = np.asarray(history).astype(np.int64).copy()
    B, V = h.shape
    for b in range(B):
        if fresh is not None and fresh[b]:
            h[b] = 0
        for t in (prompts[b] if prompts is not None else ()):
            if 0 <= t < V:
                h[b, t] |= 1
        for t in (emitted[b] if emitted is not None else ()):
            if 0 <= t < V and h[b, t] // 2 < MOST:
                h[b, t] += 2
    return h
