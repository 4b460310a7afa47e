"""Attention within a window, over 8-bit caches and for trees of drafted tokens, from the definitions, in numpy and float64."""
import numpy as np


def window_seen(n_q, n_k, batch, window=None, sinks=0, causal=True, k_len=None, q_pos=None):
    """bool [batch, n_q, n_k]: the keys that a row sees."""
    out = np.zeros((batch, n_q, n_k), dtype=bool)
    key = np.arange(n_k, dtype=np.int64)
    for b in range(batch):
        length = n_k if k_len is None else min(max(int(k_len[b]), 0), n_k)
        for i in range(n_q):
            p = (length - n_q if q_pos is None else int(q_pos[b])) + i
            if causal:
                see = (key <= p) & ((key > p - window) | (key < sinks)) if window else key <= p
            else:
                see = (key > p - window) & (key < p + window) | (key < sinks) if window else np.ones(n_k, dtype=bool)
            out[b, i] = see & (key < length)
    return out


def tree_lines(parent):
    """(ancestors of every token from the root on, itself last; depths).  What is not a token ahead of t stands for the newest committed one."""
    lines = []
    for t, up in enumerate(parent):
        lines.append((lines[int(up)] if 0 <= int(up) < t else []) + [t])
    return lines, [len(line) - 1 for line in lines]


def tree_seen(parent, n_k, window=None, sinks=0, k_len=None):
    """bool [batch, n_q, n_k] for parent [batch, n_q]: the keys that a drafted token sees."""
    batch, n_q = np.shape(parent)
    out = np.zeros((batch, n_q, n_k), dtype=bool)
    for b in range(batch):
        length = n_k if k_len is None else min(max(int(k_len[b]), 0), n_k)
        base = length - n_q
        lines, depth = tree_lines(parent[b])
        for t in range(n_q):
            at = {j: j for j in range(max(base, 0))}                          # key row -> position
            at.update({base + a: base + depth[a] for a in lines[t] if base + a >= 0})
            for row, p in at.items():
                if not window or base + depth[t] - p < window or p < sinks:
                    out[b, t, row] = True
    return out


def e4m3(x):
    """The nearest of the values that 1 + 4 + 3 bits hold, ties to even; |x| <= 448, what is not finite is NaN."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    v = np.where(fine, x, 0.0)
    step = 2.0 ** (np.maximum(np.frexp(v)[1] - 1, -6) - 3)
    return np.where(fine, np.rint(v / step) * step, np.nan)


def quantise(x, half=False):
    """(values, scales) of rows in 8 bits: the least power of two, from 2^-126 on, with max |x| <= 448 s; 1 for rows of zeros.  Of half: what would become
    256 2^8, which half does not hold, 240 2^8."""
    x = np.asarray(x, dtype=np.float64)
    most = np.where(np.isfinite(x), np.abs(x), 0.0).max(-1)
    power = np.zeros(most.shape, dtype=np.int64)
    for at in np.ndindex(most.shape):
        if most[at] > 0:
            power[at] = -126
            while most[at] > 448 * 2.0 ** power[at]:
                power[at] += 1
    s = 2.0 ** power
    if half:
        x = np.where((s[..., None] == 256) & (np.abs(x) < 65520), np.clip(x, -240 * 256, 240 * 256), x)
    return e4m3(x / s[..., None]), s
