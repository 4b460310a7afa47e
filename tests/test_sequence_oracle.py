"""The float64 oracle of the token-sequence operators against loops over single numbers and closed forms (CPU)."""
import math

import numpy as np

from oracle import sequence_oracle as orc


def test_rotation_is_a_complex_product_and_keeps_distances():
    gen = np.random.default_rng(1)
    x, f = gen.standard_normal((5, 16)), orc.rotary_frequencies(4)
    angle = np.arange(5)[:, None] * f
    y = orc.rotary(x, angle, 1.0, "half")
    z = (x[:, :4] + 1j * x[:, 4:8]) * np.exp(1j * angle)
    assert np.allclose(y[:, :4], z.real) and np.allclose(y[:, 4:8], z.imag) and np.array_equal(y[:, 8:], x[:, 8:])
    w = orc.rotary(x, angle, 1.0, "interleaved")
    z = (x[:, 0:8:2] + 1j * x[:, 1:8:2]) * np.exp(1j * angle)
    assert np.allclose(w[:, 0:8:2], z.real) and np.allclose(w[:, 1:8:2], z.imag)
    assert np.allclose(orc.rotary(y, angle, 1.0, "half", inverse=True), x)
    # the product of two turned rows goes by the distance of their positions only
    q, k = x[0], x[1]
    dots = [orc.rotary(q, (n + 3) * f, 1.0, "half") @ orc.rotary(k, n * f, 1.0, "half") for n in (0, 5, 100)]
    assert np.allclose(dots, dots[0])


def test_frequencies():
    f = orc.rotary_frequencies(8, base=10000.0)
    assert f[0] == 1.0 and math.isclose(f[4], 0.01)
    assert np.allclose(orc.rotary_frequencies(8, scaling="linear", factor=4.0), f / 4)
    g = orc.rotary_frequencies(8, scaling="base", factor=4.0)
    assert g[0] == 1.0 and math.isclose(g[-1], f[-1] / 4)
    r = orc.rotary_frequencies(64, scaling="ramp", factor=8.0, trained=4096.0, low=1.0, high=32.0)
    f = orc.rotary_frequencies(64)
    turns = 4096 * f / (2 * math.pi)
    assert np.array_equal(r[turns >= 32], f[turns >= 32]) and np.allclose(r[turns <= 1], f[turns <= 1] / 8)
    assert (np.diff(r) < 0).all()


def test_rows_see():
    see = orc.rows_see(3, 5, 2, True, k_len=[5, 2])
    assert see[0].sum(1).tolist() == [3, 4, 5] and see[1].sum(1).tolist() == [0, 1, 2]
    assert orc.rows_see(3, 5, 1, False, k_len=[2])[0].sum(1).tolist() == [2, 2, 2]
    assert orc.rows_see(2, 5, 1, True, q_pos=[-1])[0].sum(1).tolist() == [0, 1]


def test_selection_by_hand():
    s = np.array([[[[0.0, 5.0, 1.0, 5.0, 2.0, 9.0]]]])
    where = dict(n_q=1, n_k=6 * 32, q_group=1, block=32, causal=True)
    assert orc.select_blocks(s, 3, 1, 1, **where)[0][0][0] == [0, 1, 5]     # of the two fives the first
    assert orc.select_blocks(s, 4, 0, 0, **where)[0][0][0] == [1, 3, 4, 5]
    assert orc.select_blocks(s, 4, 0, 1, k_len=[70], **where)[0][0][0] == [0, 1, 2]   # three blocks are seen
    s[..., 1], s[..., 3] = np.nan, -np.inf
    assert orc.select_blocks(s, 6, 0, 0, **where)[0][0][0] == [0, 2, 4, 5]


def brute(Q, K, V, scale, mask):
    B, H, N, d = Q.shape
    O, lse = np.zeros_like(Q), np.full((B, H, N), -math.inf)
    share = H // K.shape[1]
    for b in range(B):
        for h in range(H):
            for i in range(N):
                w = {j: math.exp(scale * sum(Q[b, h, i, c] * K[b, h // share, j, c] for c in range(d)))
                     for j in range(K.shape[2]) if mask[b, h // share, i, j]}
                if w:
                    total = sum(w.values())
                    lse[b, h, i] = math.log(total)
                    for j, e in w.items():
                        O[b, h, i] += e / total * V[b, h // share, j]
    return O, lse


def test_attention_and_its_gradient_against_loops_and_differences():
    gen = np.random.default_rng(2)
    B, Hq, Hkv, N, M, d, q_group, block = 2, 4, 2, 5, 9, 4, 2, 3
    Q, K, V = (gen.standard_normal((B, h, n, d)) for h, n in ((Hq, N), (Hkv, M), (Hkv, M)))
    index = gen.permuted(np.broadcast_to(np.arange(3), (B, Hkv, 3, 3)), axis=-1)[..., :2].copy()
    count = gen.integers(0, 3, (B, Hkv, 3))
    mask = orc.attended(count, index, N, M, q_group, block, True, k_len=[9, 6])
    assert not mask.any(-1).all()            # rows that attend nothing are among them
    O, lse, P = orc.attention(Q, K, V, 0.6, mask)
    Ob, lb = brute(Q, K, V, 0.6, mask)
    assert np.allclose(O, Ob, atol=1e-12) and np.allclose(lse, lb, atol=1e-12)
    dO = gen.standard_normal(O.shape)
    grads = orc.attention_gradient(dO, Q, K, V, 0.6, mask)
    for x, g in zip((Q, K, V), grads):
        for _ in range(12):
            at = tuple(gen.integers(0, n) for n in x.shape)
            keep, e = x[at], 1e-5
            x[at] = keep + e
            hi = (orc.attention(Q, K, V, 0.6, mask)[0] * dO).sum()
            x[at] = keep - e
            lo = (orc.attention(Q, K, V, 0.6, mask)[0] * dO).sum()
            x[at] = keep
            assert abs((hi - lo) / (2 * e) - g[at]) < 1e-8
