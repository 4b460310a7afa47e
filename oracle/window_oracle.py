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
