"""Token sequences in float64 numpy, from the definitions: rotary positions, block means and scores, selection, attention over
lists of key blocks and its gradient.  Shares no code with the GPU side; every mask is built key by key."""
import math

import numpy as np


def rotary_frequencies(pairs, base=10000.0, scaling="plain", factor=1.0, trained=0.0, low=1.0, high=32.0):
    """Radians per position of one axis' pairs."""
    if scaling == "base" and pairs > 1:
        base = base * factor ** (pairs / (pairs - 1))
    f = np.array([base ** (-i / pairs) for i in range(pairs)])
    if scaling == "linear":
        f = f / factor
    if scaling == "ramp":
        w = np.clip((trained * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        f = f * (w + (1 - w) / factor)
    return f


def rotary(x, angle, magnitude, layout, inverse=False):
    """x [..., d] turned by angle [..., pairs] (broadcast): each pair times the 2x2 rotation matrix."""
    y = np.array(x, dtype=np.float64)
    pairs = angle.shape[-1]
    for p in range(pairs):
        a, b = (2 * p, 2 * p + 1) if layout == "interleaved" else (p, p + pairs)
        c, s = magnitude * np.cos(angle[..., p]), magnitude * np.sin(angle[..., p])
        if inverse:
            s = -s
        y[..., a], y[..., b] = c * x[..., a] - s * x[..., b], s * x[..., a] + c * x[..., b]
    return y


def positions(n_q, n_k, batch, k_len=None, q_pos=None):
    """(valid keys, position of every query row) of every sequence."""
    length = [min(max(int(k_len[b]), 0), n_k) if k_len is not None else n_k for b in range(batch)]
    first = [int(q_pos[b]) if q_pos is not None else length[b] - n_q for b in range(batch)]
    return length, [[f + i for i in range(n_q)] for f in first]


def rows_see(n_q, n_k, batch, causal, k_len=None, q_pos=None):
    """bool [batch, n_q, n_k]: the keys that a row sees."""
    length, at = positions(n_q, n_k, batch, k_len, q_pos)
    see = np.zeros((batch, n_q, n_k), dtype=bool)
    for b in range(batch):
        keys = np.arange(n_k)
        for i in range(n_q):
            see[b, i] = (keys < length[b]) & ((keys <= at[b][i]) if causal else True)
    return see


def block_means(K, block, k_len=None):
    B, H, M, d = K.shape
    blocks = -(-M // block)
    out = np.zeros((B, H, blocks, d))
    for b in range(B):
        n = min(max(int(k_len[b]), 0), M) if k_len is not None else M
        for j in range(-(-n // block)):
            out[b, :, j] = K[b, :, j * block:min(n, (j + 1) * block)].astype(np.float64).mean(1)
    return out


def blocks_seen(n_q, n_k, batch, q_group, block, causal, k_len=None, q_pos=None):
    """int [batch, groups]: blocks [0, s) hold every key that a row of the group sees."""
    see = rows_see(n_q, n_k, batch, causal, k_len, q_pos)
    groups = -(-n_q // q_group)
    out = np.zeros((batch, groups), dtype=int)
    for b in range(batch):
        for g in range(groups):
            keys = np.nonzero(see[b, g * q_group:(g + 1) * q_group].any(0))[0]
            out[b, g] = 0 if keys.size == 0 else keys[-1] // block + 1
    return out


def block_scores(Q, means, scale, q_group, block, n_k, causal, k_len=None, q_pos=None):
    B, Hq, N, d = Q.shape
    Hkv, blocks = means.shape[1], means.shape[2]
    share, groups = Hq // Hkv, -(-N // q_group)
    seen = blocks_seen(N, n_k, B, q_group, block, causal, k_len, q_pos)
    out = np.full((B, Hkv, groups, blocks), -np.inf)
    for b in range(B):
        for h in range(Hkv):
            for g in range(groups):
                q = Q[b, h * share:(h + 1) * share, g * q_group:(g + 1) * q_group].astype(np.float64).reshape(-1, d).mean(0)
                n = seen[b, g]
                out[b, h, g, :n] = scale * (means[b, h, :n].astype(np.float64) @ q)
    return out


def select_blocks(scores, top, first, local, n_q, n_k, q_group, block, causal, k_len=None, q_pos=None):
    """Python lists of blocks, [B][Hkv][groups]."""
    B, Hkv, groups, _ = scores.shape
    seen = blocks_seen(n_q, n_k, B, q_group, block, causal, k_len, q_pos)
    out = []
    for b in range(B):
        out.append([])
        for h in range(Hkv):
            out[b].append([])
            for g in range(groups):
                n = int(seen[b, g])
                chosen = {j for j in range(n) if j < first or j >= n - local}
                rest = [j for j in range(n) if j not in chosen and scores[b, h, g, j] > -np.inf]   # (False for NaN)
                rest.sort(key=lambda j: (-float(scores[b, h, g, j]), j))
                chosen |= set(rest[:max(0, top - len(chosen))])
                out[b][h].append(sorted(chosen))
    return out


def attended(count, index, n_q, n_k, q_group, block, causal, k_len=None, q_pos=None):
    """bool [B, Hkv, n_q, n_k]: the listed keys that a row sees."""
    B, Hkv, groups, top = index.shape
    see = rows_see(n_q, n_k, B, causal, k_len, q_pos)
    mask = np.zeros((B, Hkv, n_q, n_k), dtype=bool)
    for b in range(B):
        for h in range(Hkv):
            for g in range(groups):
                rows = slice(g * q_group, min(n_q, (g + 1) * q_group))
                for t in range(min(max(int(count[b, h, g]), 0), top)):
                    j = int(index[b, h, g, t])
                    if 0 <= j * block < n_k:
                        keys = slice(j * block, min(n_k, (j + 1) * block))
                        mask[b, h, rows, keys] = see[b, rows, keys]
    return mask


def attention(Q, K, V, scale, mask):
    """(O, lse, P) over mask [B, Hkv, n_q, n_k]; rows that attend nothing: 0, -inf, 0."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    B, Hq, N, d = Q.shape
    share = Hq // K.shape[1]
    O, lse = np.zeros_like(Q), np.full((B, Hq, N), -np.inf)
    P = np.zeros((B, Hq, N, K.shape[2]))
    for b in range(B):
        for h in range(Hq):
            m = mask[b, h // share]
            keys = m.any(0)   # (what lies in keys that nobody attends must not count: it may be NaN)
            Kh, Vh = (np.where(keys[:, None], x[b, h // share], 0.0) for x in (K, V))
            s = np.where(m, scale * (Q[b, h] @ Kh.T), -np.inf)
            some = m.any(1)
            top = np.where(some, s.max(1, initial=-np.inf), 0.0)
            e = np.exp(s - top[:, None])
            total = e.sum(1)
            P[b, h] = e / np.where(some, total, 1.0)[:, None]
            O[b, h] = P[b, h] @ Vh
            with np.errstate(divide="ignore"):
                lse[b, h] = np.where(some, top + np.log(np.where(some, total, 1.0)), -np.inf)
    return O, lse, P


def attention_gradient(dO, Q, K, V, scale, mask):
    dO, Q, K, V = (np.asarray(x, dtype=np.float64) for x in (dO, Q, K, V))
    O, _, P = attention(Q, K, V, scale, mask)
    share = Q.shape[1] // K.shape[1]
    dQ, dK, dV = np.zeros_like(Q), np.zeros_like(K), np.zeros_like(V)
    for b in range(Q.shape[0]):
        for h in range(Q.shape[1]):
            g = h // share
            keys = mask[b, g].any(0)[:, None]
            Kh, Vh = np.where(keys, K[b, g], 0.0), np.where(keys, V[b, g], 0.0)
            dP = dO[b, h] @ Vh.T
            dS = P[b, h] * (dP - (dO[b, h] * O[b, h]).sum(1, keepdims=True)) * scale
            dQ[b, h] = dS @ Kh
            dK[b, g] += dS.T @ Q[b, h]
            dV[b, g] += P[b, h].T @ dO[b, h]
    return dQ, dK, dV
