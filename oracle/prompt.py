"""fp64 oracle of what a prompt passes through: rotary positions and causal attention of packed sequences."""
from __future__ import annotations

import math

import numpy as np


def frequencies(rot, base, scaling="none", factor=1.0, low=1.0, high=32.0, original=8192.0):
    """Radians a position of every pair, and the amplitude: one pair after the other, from the definitions."""
    f, amplitude = [], 1.0
    for i in range(rot // 2):
        w = base ** (-2.0 * i / rot)
        if scaling == "linear":
            w = w / factor
        elif scaling == "bands":
            turns = original * w / (2 * math.pi)               # within the original length
            if turns <= low:
                w = w / factor
            elif turns < high:
                part = (turns - low) / (high - low)
                w = part * w + (1 - part) * w / factor
        elif scaling == "yarn":
            def pair(turns):                                   # the pair, as a real number, that turns so often
                return rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))
            first, last = max(math.floor(pair(high)), 0), min(math.ceil(pair(low)), rot - 1)
            part = min(max((i - first) / max(last - first, 1e-3), 0.0), 1.0)
            w = (1 - part) * w + part * w / factor
            amplitude = 0.1 * math.log(factor) + 1.0
        f.append(w)
    return np.array(f), amplitude


def depth(parents, node):
    """Steps from a tree's node to its root; a parent that is not an earlier node counts as the root."""
    n = 0
    while node > 0:
        p = parents[node - 1]
        node = p if 0 <= p < node else 0
        n += 1
    return n


def rotate(x, positions, f, amplitude, interleaved):
    """x [T, H, d] fp64 rotated to positions [T]; rows with a negative one come back as they are."""
    x, half = np.asarray(x, np.float64), len(f)
    y = x.copy()
    for t, pos in enumerate(positions):
        if pos < 0:
            continue
        z = amplitude * np.exp(1j * (float(pos) * f))
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        w = (x[t, :, a] + 1j * x[t, :, b]) * z
        y[t, :, a], y[t, :, b] = w.real, w.imag
    return y


def attention(q, k, v, cu, scale):
    """out [T, Hq, d], and sum_j p_j |v_j|, the size that errors of the probabilities scale with.  Rows of no sequence: zeros."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    T, Hq, _ = q.shape
    G = Hq // k.shape[1]
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for lo, hi in zip(cu[:-1], cu[1:]):
        for h in range(Hq):
            for i in range(lo, hi):
                s = scale * (k[lo:i + 1, h // G] @ q[i, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[i, h] = p @ v[lo:i + 1, h // G]
                size[i, h] = p @ np.abs(v[lo:i + 1, h // G])
    return out, size
