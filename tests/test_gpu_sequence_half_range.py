"""The gradient of attention over lists in half, for dO and V of every size, vs the float64 oracle.

Bounds as in test_gpu_sequence_attention.py, but for dS: it is rounded to half times a power of two, so what half's subnormal numbers cost is
   2^-25 / 2^k   with  |dO| 2^k >= 2^9 of the row (dQ), and >= 2^8 of the K/V head's largest row (dK); 2^16 times as much where V is so large that dS
   would leave half at that size, |V| > 2^6 (the largest |dS| is |dO| |V| / 2 or less: P (1 - P) times a difference of two V)."""
import math

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle as orc
from sequence_util import f64, ints, normal
from test_gpu_sequence_attention import random_lists, within

pytestmark = pytest.mark.gpu
EPS, U, TINY = 2.0 ** -24, 2.0 ** -11, 2.0 ** -25

SHAPES = [   # B, Hq, Hkv, N, M, q_group, block, top, k_len
    (2, 8, 2, 45, 500, 1, 64, 6, [500, 90]),       # 4 rows a list, 12 units
    (1, 3, 1, 60, 900, 4, 32, 20, None),           # 12 rows, 20 units
    (2, 4, 4, 100, 100, 32, 32, 4, None),          # 32 rows
    (1, 4, 2, 130, 1100, 32, 64, 12, None),        # 64 rows, 24 units
    (2, 4, 1, 200, 200, 48, 64, 4, [200, 150]),    # 192 rows, 8 units
    (1, 8, 2, 260, 1500, 64, 64, 16, None),        # 256 rows, 32 units
    (1, 1, 1, 3000, 300, 1, 32, 3, None),          # lists turned round through memory
]


def bounds(dO, Q, K, V, scale, mask, back):
    O, _, P = orc.attention(Q, K, V, scale, mask)
    B, Hq, N, d = Q.shape
    share = Hq // K.shape[1]
    keys = mask.any(2)[..., None]
    K, V = np.where(keys, K, 0.0), np.where(keys, V, 0.0)
    n = max(1, int(mask.sum(-1).max()))
    grads, lims = [np.zeros_like(x) for x in (Q, K, V)], [np.zeros_like(x) for x in (Q, K, V)]
    for b in range(B):
        for g in range(K.shape[1]):
            k, v = K[b, g], V[b, g]
            heads = range(g * share, (g + 1) * share)
            largest = max(np.linalg.norm(dO[b, h], axis=1)[mask[b, g].any(1)].max(initial=0.0) for h in heads)
            for h in heads:
                q, p, do = Q[b, h], P[b, h], dO[b, h]
                w = (d + 8) * EPS * scale * (np.abs(q) @ np.abs(k).T).max(initial=0) + n * EPS
                bO = U * (p @ np.abs(v)) + U * np.abs(O[b, h]) + 4 * w * (p @ np.abs(v)) + TINY
                ds = p * (do @ v.T - (do * O[b, h]).sum(1, keepdims=True))
                E = p * ((d + 1) * EPS * (np.abs(do) @ np.abs(v).T) + (np.abs(do) * (bO + d * EPS * np.abs(O[b, h]))).sum(1, keepdims=True))
                bs = (U + 4 * w) * np.abs(ds) + E
                row = TINY * 2.0 ** (back - 9) * np.linalg.norm(do, axis=1, keepdims=True) * mask[b, g]
                head = TINY * 2.0 ** (back - 8) * largest * mask[b, g]
                grads[0][b, h] = scale * (ds @ k)
                lims[0][b, h] = scale * ((bs + row + n * EPS * np.abs(ds)) @ np.abs(k))
                grads[1][b, g] += scale * (ds.T @ q)
                lims[1][b, g] += scale * ((bs + head + N * share * EPS * np.abs(ds)).T @ np.abs(q))
                grads[2][b, g] += p.T @ do
                lims[2][b, g] += ((U + 4 * w + N * share * EPS) * p.T + 2.0 ** -12 * TINY * mask[b, g].T) @ np.abs(do)
    return grads, [x + U * np.abs(g) + TINY for x, g in zip(lims, grads)]


def run(shape, d, gains, seed, rows=None):
    """gains of dO, Q, K, V; rows: a factor for every sequence, head and row of dO."""
    B, Hq, Hkv, N, M, q_group, block, top, k_len = shape
    gen = np.random.default_rng(seed)
    count, index = random_lists(gen, B, Hkv, -(-N // q_group), -(-M // block), top, full=True)
    dO, Q = (normal((B, Hq, N, d), "f16", seed + i, "tokens", gain) for i, gain in enumerate(gains[:2]))
    K, V = (normal((B, Hkv, M, d), "f16", seed + 2 + i, "heads", gain) for i, gain in enumerate(gains[2:]))
    if rows is not None:
        dO = (dO.float() * rows(gen, (B, Hq, N, 1))).half()
    scale = 1 / math.sqrt(d)
    args = dict(q_group=q_group, block=block, k_len=ints(k_len))
    lists = torch.from_numpy(count).cuda(), torch.from_numpy(index).cuda()
    O, lse = grat.grat_selected_attention_fwd(Q, K, V, scale, *lists, return_lse=True, **args)
    grads = grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, scale, *lists, **args)
    mask = orc.attended(count, index, N, M, q_group, block, True, k_len)
    want, lims = bounds(*(f64(t) for t in (dO, Q, K, V)), scale, mask, 16 if gains[3] >= 8 else 0)
    for name, got, w, lim in zip(("dQ", "dK", "dV"), grads, want, lims):
        got = f64(got)
        beyond = np.abs(w) + lim >= 65520.0          # (rounds to infinity)
        assert (np.isfinite(got) | beyond & (np.sign(got) == np.sign(w))).all(), f"{name}: not finite"
        within(np.where(beyond & np.isinf(got), w, got), w, lim, name)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("gains", [
    (2.0 ** -13, 1 / 32, 32, 1),      # small gradients; dQ itself is not small
    (2.0 ** -13, 32, 1 / 32, 1),      # ... and dK
    (2.0 ** -10, 1, 1, 2.0 ** -4),
    (2.0 ** 10, 8, 0.25, 4),          # |dS| beyond 65 504 where dQ is not
    (2.0 ** 10, 0.25, 8, 4),          # ... where dK is not
    (1, 1, 1, 512),                   # large V: rows are walked again
    (2.0 ** -8, 2, 2, 4096),
])
def test_sizes(d, shape, gains):
    run(shape, d, gains, 300)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_rows_of_different_sizes(d, shape):
    """Sequences 2^10 apart, rows of a sequence up to 2^6, and rows of zeros."""
    def rows(gen, s):
        f = 2.0 ** -gen.integers(0, 7, s).astype(np.float64) * (gen.random(s) < 0.8)
        f[1:] *= 2.0 ** -10
        return torch.tensor(f, dtype=torch.float32, device="cuda")
    run(shape, d, (1, 1, 1, 1), 310, rows)


def test_no_gradient_at_all():
    shape = SHAPES[3]
    run(shape, 128, (1, 1, 1, 1), 320, lambda gen, s: torch.zeros(s, device="cuda"))


def test_a_graph_follows_the_size_of_dO():
    """Replays of a recorded step with dO of other sizes, between other work: the exponents belong to the replay."""
    B, Hq, Hkv, N, M, q_group, block, top, k_len = SHAPES[4]
    count, index = random_lists(np.random.default_rng(330), B, Hkv, -(-N // q_group), -(-M // block), top, full=True)
    lists = torch.from_numpy(count).cuda(), torch.from_numpy(index).cuda()
    args, scale = dict(q_group=q_group, block=block, k_len=ints(k_len)), 0.125
    Q, K, V = (normal((B, h, n, 64), "f16", 331 + i) for i, (h, n) in enumerate(((Hq, N), (Hkv, M), (Hkv, M))))
    sizes = [normal((B, Hq, N, 64), "f16", 340 + i, gain=gain) for i, gain in enumerate((1.0, 2.0 ** -13, 2.0 ** 9))]
    O, lse = grat.grat_selected_attention_fwd(Q, K, V, scale, *lists, return_lse=True, **args)

    def step(dO):
        return grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, scale, *lists, **args)
    eager = [step(dO) for dO in sizes]
    static = sizes[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(static)
    for i in (0, 1, 2, 1, 0):
        static.copy_(sizes[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, eager[i])), f"replay with dO {i}"
        step(sizes[(i + 1) % 3])
