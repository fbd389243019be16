"""The key / value cache of a round, written out plainly in 64 bits: a stack of free blocks popped and pushed
sequence by sequence, e4m3 as a table of its 256 values, softmax over the positions a token sees."""
from __future__ import annotations

import numpy as np

BAD_LENGTH, NO_BLOCKS, NO_ROOM = 64, 128, 256


# ---- e4m3 ----------------------------------------------------------------------------------

def e4m3_values() -> np.ndarray:
    """Value of every code: sign, 4 exponent bits (bias 7), 3 significand bits; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        s, e, m = c >> 7, (c >> 3) & 15, c & 7
        x = (m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7)
        v[c] = np.nan if e == 15 and m == 7 else (-x if s else x)
    return v


VALUES = e4m3_values()


def encode(x: np.ndarray) -> np.ndarray:
    """Nearest code, ties to the even code, too large to +-448, NaN to a NaN code."""
    x = np.asarray(x, dtype=np.float64)
    pos = VALUES[:127]                                    # ascending, 0 .. 448
    a = np.minimum(np.abs(x), 448.0)
    hi = np.clip(np.searchsorted(pos, a, side="left"), 0, 126)
    lo = np.maximum(hi - 1, 0)
    d_hi, d_lo = pos[hi] - a, a - pos[lo]
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (hi % 2 == 0))
    c = np.where(up, hi, lo).astype(np.uint8)
    c = np.where(np.signbit(x), c | 0x80, c)
    return np.where(np.isnan(x), np.uint8(0x7F), c).astype(np.uint8)


def block_scale(x: np.ndarray) -> float:
    """The smallest power of two >= 2^-64 that brings the largest finite magnitude to 448 or less."""
    f = np.abs(x[np.isfinite(x)])
    amax = float(f.max()) if f.size else 0.0
    s = 2.0 ** -64
    while amax > 448.0 * s:
        s *= 2.0
    return s


# ---- plan ------------------------------------------------------------------------------------

def plan(seq_len, kept, n_new, extra, active, bt, table, held, free, T, last_cu=None, shared=None):
    """One call.  `free`: list, its top last.  last_cu: cu_new of the call whose tokens `kept` counts.  shared: leading
    blocks of every sequence that are not returned.  Returns the new state and the outputs as a dict."""
    if kept is not None and last_cu is not None:
        got = np.diff(last_cu)
        kept = [k if k <= 0 else 0 if g <= 0 else -1 if k > g else k for k, g in zip(np.asarray(kept).tolist(), got.tolist())]
    B, W = table.shape
    seq_len, table, held, free = seq_len.copy(), table.copy(), held.copy(), list(free)
    status, new, kv = np.zeros(B, np.int64), np.zeros(B, np.int64), np.zeros(B, np.int64)
    want = held.astype(np.int64).copy()
    asked = 0
    for b in range(B):
        on = active is None or active[b]
        L = int(seq_len[b]) + (int(kept[b]) if on and kept is not None else 0)
        n = int(n_new[b]) + extra if on else 0
        sh = 0 if shared is None else int(shared[b])
        if seq_len[b] < 0 or (on and kept is not None and kept[b] < 0) or n < 0 or not 0 <= held[b] <= W \
                or L > held[b] * bt or L + n > W * bt or not 0 <= sh <= held[b] or (n > 0 and L < sh * bt):
            status[b] = BAD_LENGTH
            continue
        asked += n
        seq_len[b], kv[b] = L, L
        if n > 0 and asked > T:
            status[b] = NO_ROOM
            continue
        new[b] = n
        want[b] = max(-(-(L + n) // bt), sh)
    gone = []                                             # surplus blocks, in the order of the sequences
    for b in range(B):
        for j in range(int(want[b]), int(held[b])):
            gone.append(table[b, j])
            table[b, j] = -1
    free += gone[::-1]                                    # the first of them ends on top
    need, avail = 0, len(free)
    for b in range(B):
        short = max(0, int(want[b]) - int(held[b]))
        need += short
        if short and need > avail:
            status[b] |= NO_BLOCKS
            new[b], want[b] = 0, held[b]
            continue
        for j in range(int(held[b]), int(want[b])):
            table[b, j] = free.pop()
    cu = np.concatenate([[0], np.cumsum(new)])
    slots, pos = np.full(T, -1, np.int64), np.full(T, -1, np.int64)
    for b in range(B):
        for i in range(int(new[b])):
            q = int(kv[b]) + i
            pos[cu[b] + i] = q
            slots[cu[b] + i] = table[b, q // bt] * bt + q % bt
    return dict(seq_len=seq_len, table=table, held=want, free=free, kv_len=kv + new, cu_new=cu, slot_map=slots,
                positions=pos, status=status)


# ---- append, keep ------------------------------------------------------------------------------

def append(x, slots, codes, scale, bt):
    """x [T, H, d] into codes [n_blocks, H, bt, d] (uint8) and scale [n_blocks, H], in place."""
    T, H, _ = x.shape
    i = 0
    while i < T:
        if slots[i] < 0 or slots[i] >= codes.shape[0] * bt:
            i += 1
            continue
        blk, off = divmod(int(slots[i]), bt)
        n = 1
        while i + n < T and off + n < bt and slots[i + n] == slots[i] + n:
            n += 1
        for h in range(H):
            rows = np.asarray(x[i:i + n, h], dtype=np.float64)
            s = block_scale(rows)
            if off:
                old = float(scale[blk, h])
                if s > old:
                    codes[blk, h, :off] = encode(VALUES[codes[blk, h, :off]] * old / s)
                s = max(s, old)
            codes[blk, h, off:off + n] = encode(rows / s)
            scale[blk, h] = s
        i += n


def keep_path(path, base, table, codes, scale, bt):
    """The accepted path (node numbers) of one sequence whose tree begins at position `base`, in place."""
    was, sc = codes.copy(), scale.copy()
    for h in range(scale.shape[1]):
        pages = {}
        for j, node in enumerate(path):
            pages.setdefault((base + 1 + j) // bt, []).append(((base + 1 + j) % bt, divmod(base + node, bt)))
        for page, moves in pages.items():
            blk = table[page]
            s = max([sc[blk, h]] + [sc[table[m[1][0]], h] for m in moves])
            lead = moves[0][0]
            codes[blk, h, :lead] = encode(VALUES[was[blk, h, :lead]] * float(sc[blk, h]) / float(s))
            for to, (sp, so) in moves:
                codes[blk, h, to] = encode(VALUES[was[table[sp], h, so]] * float(sc[table[sp], h]) / float(s))
            scale[blk, h] = s


# ---- attention ----------------------------------------------------------------------------------

def sees(n, base, parent=None):
    """[n, base + n] which positions each new token sees; parent[k - 1] = parent of node k of a tree."""
    m = np.zeros((n, max(0, base + n)), dtype=bool)
    for i in range(n):
        if parent is None:
            m[i, :max(0, base + i + 1)] = True
            continue
        m[i, :max(0, base)] = True
        k = i
        while True:
            if base + k >= 0:
                m[i, base + k] = True
            if k == 0:
                break
            p = int(parent[k - 1])
            k = p if 0 <= p < k else 0
    return m


def attention(q, blocks, kv_len, k_codes, k_scale, v_codes, v_scale, softmax_scale, parent=None):
    """q [n, Hq, d] of one sequence; blocks: its row of the block table.  Returns [n, Hq, d]."""
    n, Hq, d = q.shape
    Hkv, bt = k_codes.shape[1], k_codes.shape[2]
    G, base = Hq // Hkv, kv_len - n
    out = np.zeros((n, Hq, d))
    see = sees(n, base, parent)
    nb = -(-kv_len // bt)
    for h in range(Hkv):
        k = (VALUES[k_codes[blocks[:nb], h]] * k_scale[blocks[:nb], h][:, None, None].astype(np.float64)).reshape(-1, d)[:kv_len]
        v = (VALUES[v_codes[blocks[:nb], h]] * v_scale[blocks[:nb], h][:, None, None].astype(np.float64)).reshape(-1, d)[:kv_len]
        for g in range(G):
            for i in range(n):
                idx = np.nonzero(see[i])[0]
                if not idx.size:
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    t = k[idx] @ q[i, h * G + g] * softmax_scale
                    e = np.exp(t - t.max())
                    out[i, h * G + g] = (e / e.sum()) @ v[idx]
    return out
