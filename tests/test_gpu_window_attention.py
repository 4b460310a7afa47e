"""Attention within a window and its gradient vs the float64 oracle; the bounds are those of test_gpu_sequence_attention.py, with the keys that a row
sees in the place of listed ones."""
import math

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import window_oracle as orc
from sequence_util import f64, ints, nan_like, normal
from test_gpu_sequence_attention import bounds, within

pytestmark = pytest.mark.gpu

# B, Hq, Hkv, N, M, window, sinks, k_len, q_pos, causal
TOKENS = [
    (1, 4, 4, 1, 1, 1, 0, None, None, True),                       # one key
    (3, 8, 2, 1, 700, 100, 5, [700, 1, 65], None, True),           # serving
    (2, 16, 1, 1, 3000, 2000, 40, [2999, 130], None, True),        # keys shared by several workgroups; a cache shorter than the window
    (2, 40, 1, 1, 900, None, 0, [900, 0], None, True),             # more heads than a row tile; an empty cache; no limit
    (1, 6, 2, 5, 400, 33, 32, None, None, True),                   # a few tokens
    (2, 8, 8, 3, 1500, 1300, 1, [1500, 2], None, True),            # rows ahead of the first key
    (1, 1, 1, 1, 1100, 1, 1024, None, None, True),                 # more first keys than window
]
PROMPTS = [
    (2, 4, 4, 100, 100, 20, 3, None, None, True),
    (2, 4, 2, 130, 130, 64, 0, [130, 70], None, True),             # a row that sees nothing, ahead of the first key
    (1, 6, 2, 300, 300, 1, 0, None, None, True),                   # every row itself
    (1, 3, 3, 257, 500, 129, 70, None, None, True),                # a chunk behind a prefix; first keys in more than one tile
    (1, 2, 1, 200, 333, None, 0, None, None, False),               # everything
    (2, 5, 1, 150, 150, 31, 1, [150, 99], None, False),            # both directions, five heads to a K/V head
    (2, 4, 1, 70, 200, 16, 2, [200, 33], [-20, 300], True),        # positions that are given: before the first key, behind the last
    (2, 4, 1, 70, 200, 16, 2, [200, 33], [-20, 300], False),
    (1, 16, 1, 33, 1000, 500, 4, [999], None, True),
    (1, 2, 2, 700, 700, 2000, 900, None, None, True),              # a window longer than the sequence, first keys as many
    (1, 80, 2, 40, 90, 50, 33, [90], None, True),                  # 40 heads to a K/V head
    (1, 150, 1, 9, 70, 20, 2, None, None, True),                   # more heads to a K/V head than a row tile has
    (1, 150, 1, 9, 70, 20, 0, [70], [64], False),                  # ... both directions, positions behind the last key
]


def tensors(shape, dtype, d, where, seed, gain=1.0):
    B, Hq, Hkv, N, M = shape[:5]
    return (normal((B, Hq, N, d), dtype, seed, where, gain), normal((B, Hkv, M, d), dtype, seed + 1, where),
            normal((B, Hkv, M, d), dtype, seed + 2, where))


def unseen(K, V, see):
    """Keys that no row sees stay unread.  (Only those: what one row of a tile sees may reach the tile's other rows.)"""
    for b in range(K.shape[0]):
        none = torch.from_numpy(~see[b].any(0)).to(K.device)
        K[b][:, none] = float("nan")
        V[b][:, none] = float("inf")


def run_case(shape, dtype, d, where="heads", gain=1.0, backward=False, seed=31, pick=None):
    B, Hq, Hkv, N, M, window, sinks, k_len, q_pos, causal = shape
    see = orc.window_seen(N, M, B, window, sinks, causal, k_len, q_pos)
    Q, K, V = tensors(shape, dtype, d, where, seed, gain)
    unseen(K, V, see)
    scale = 1.0 / math.sqrt(d)
    args = dict(window=window, sinks=sinks, causal=causal, k_len=ints(k_len), q_pos=ints(q_pos))
    out = nan_like(Q)
    O, lse = grat.grat_window_attention_fwd(Q, K, V, scale, return_lse=True, out=out, **args)
    assert O is out
    assert torch.equal(O, grat.grat_window_attention_fwd(Q, K, V, scale, **args))
    dO = normal((B, Hq, N, d), dtype, seed + 5, where) if backward else None
    if backward:
        grads = tuple(nan_like(t) for t in (Q, K, V))
        grat.grat_window_attention_bwd(dO, Q, K, V, O, lse, scale, out=grads, **args)
        twice = grat.grat_window_attention_bwd(dO, Q, K, V, O, lse, scale, **args)
        assert all(torch.equal(x, y) for x, y in zip(grads, twice))
    share = Hq // Hkv
    for b, h in pick or [(slice(0, B), slice(0, Hkv))]:
        b, h = (slice(b, b + 1) if isinstance(b, int) else b), (slice(h, h + 1) if isinstance(h, int) else h)
        hq = slice(h.start * share, h.stop * share)
        mask = np.repeat(see[b][:, None], h.stop - h.start, 1)
        with np.errstate(invalid="ignore"):
            Ow, lw, bO, bl, gw, bG = bounds(f64(Q[b, hq]), f64(K[b, h]), f64(V[b, h]), scale, mask, dtype, f64(dO[b, hq]) if backward else None)
        within(f64(O[b, hq]), Ow, bO, "O")
        got = f64(lse[b, hq])
        assert np.array_equal(np.isneginf(got), np.isneginf(lw)), "rows that see nothing"
        fin = np.isfinite(lw)
        within(got[fin], lw[fin], bl[fin], "lse")
        if backward:
            for name, t, w, lim, head in zip(("dQ", "dK", "dV"), grads, gw, bG, (hq, h, h)):
                within(f64(t[b, head]), w, lim, name)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("shape", TOKENS + PROMPTS)
def test_forward(dtype, d, shape):
    run_case(shape, dtype, d, where="tokens" if d == 128 else "wide")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("shape", TOKENS + PROMPTS)
def test_gradient(dtype, d, shape):
    run_case(shape, dtype, d, where="wide" if d == 128 else "tokens", backward=True, seed=41)


@pytest.mark.parametrize("dtype,gain", [("bf16", 16.0), ("f16", 8.0)])
@pytest.mark.parametrize("shape", [TOKENS[1], PROMPTS[1], PROMPTS[3], PROMPTS[5]])
def test_peaked_weights(dtype, gain, shape):
    """Scores far apart: the reference maximum is refreshed on the way."""
    run_case(shape, dtype, 128, gain=gain, backward=True, seed=51)


@pytest.mark.parametrize("shape,dtype,pick", [
    ((1, 8, 2, 2100, 2100, 300, 4, None, None, True), "bf16", [(0, 1)]),
    ((1, 4, 4, 1500, 1500, 700, 100, None, None, False), "f16", [(0, 3)]),
    ((1, 4, 1, 1500, 3000, None, 0, None, None, True), "bf16", None),
    ((4, 32, 8, 2047, 2047, 200, 3, [2047, 1500, 70, 0], None, True), "bf16", [(0, 0), (1, 6), (2, 7), (3, 2)]),   # many workgroups
    ((4, 32, 32, 2700, 2700, None, 0, [2700, 1500, 70, 0], None, True), "bf16", [(0, 0), (1, 30), (2, 7), (3, 2)]),                # of 256 rows
    ((2, 12, 4, 11000, 600, 80, 5, None, [0, 30], True), "f16", [(1, 2)]),                                        # more queries than keys
])
def test_larger(shape, dtype, pick):
    run_case(shape, dtype, 128, where="tokens", backward=True, seed=61, pick=pick)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("shape,pick", [
    ((16, 32, 32, 100, 130, 20, 3, None, None, True), [(0, 0), (7, 31), (15, 5)]),           # many short prompts: 128 rows
    ((16, 32, 32, 100, 130, 20, 3, [130] * 8 + [40] * 8, None, False), [(0, 0), (15, 5)]),
    ((1, 2, 1, 150, 2700, 2650, 3, None, None, True), None),                                 # a chunk on many keys
    ((1, 1, 1, 250, 2000, 300, 2, [1700], None, True), None),                                # 250 rows that see different keys
    ((1, 1, 1, 250, 3000, 990, 2, None, None, True), None),                                  # ... in several parts
    ((1, 4, 1, 60, 4000, 1000, 2, None, None, True), None),                                  # 240 rows that see the same
])
def test_tiles_of_rows(shape, pick, dtype, d):
    run_case(shape, dtype, d, where="tokens", backward=True, seed=71, pick=pick)


def test_gradient_against_differences():
    """Directional differences of sum(O dO) in the kernels' own forward pass, in half; the bound as for attention over lists."""
    shape = (1, 2, 1, 40, 90, 20, 5, None, None, True)
    gen = np.random.default_rng(81)
    Q, K, V = tensors(shape, "f16", 64, "heads", 82)
    dO = normal((1, 2, 40, 64), "f16", 85)
    args = dict(window=20, sinks=5)

    def value(q, k, v):
        return float((grat.grat_window_attention_fwd(q, k, v, 0.125, **args).double() * dO.double()).sum())

    step = 2.0 ** -5
    for i in range(3):
        base = [Q, K, V]
        base[i] = x = torch.round(base[i] * 256) / 256          # (so that x + step is exact in half)
        O, lse = grat.grat_window_attention_fwd(*base, 0.125, return_lse=True, **args)
        g = grat.grat_window_attention_bwd(dO, *base, O, lse, 0.125, **args)[i]
        sign = torch.from_numpy(gen.choice([-1.0, 1.0], tuple(x.shape))).to(x)
        lo, hi = list(base), list(base)
        lo[i], hi[i] = x - step * sign, x + step * sign
        slope = (value(*hi) - value(*lo)) / (2 * step)
        want, size = float((g.double() * sign.double()).sum()), float(g.double().norm())
        noise = math.sqrt(2 * O.numel()) * 2.0 ** -11 * float(O.double().square().mean().sqrt()) / (2 * step)
        assert abs(slope - want) <= 6 * noise + step * size, (i, slope, want, noise, size)


@pytest.mark.parametrize("n", [40, 9000])
def test_agrees_with_lists(n):
    """A window that covers everything is what lists of all blocks attend."""
    Q, K, V = tensors((1, 4, 2, n, n), "bf16", 128, "tokens", 95)
    if n > 1000:
        Q = Q[:, :, -50:]
    blocks = -(-n // 64)
    index = torch.arange(blocks, dtype=torch.int32, device="cuda").expand(1, 2, 1, blocks).contiguous()
    count = torch.full((1, 2, 1), blocks, dtype=torch.int32, device="cuda")
    want = grat.grat_selected_attention_fwd(Q, K, V, 0.09, count, index, Q.shape[2], 64)
    for window in (None, n, 2 ** 31 - 1):
        got = grat.grat_window_attention_fwd(Q, K, V, 0.09, window=window)
        assert torch.allclose(got.double(), want.double(), rtol=2.0 ** -6, atol=2.0 ** -9)   # (each off by 2 u = 2^-7 of P |V|)


def test_offsets_beyond_32_bits():
    """A cache whose rows lie beyond 4 GiB (and whose element offsets pass 2^31)."""
    M, d = (1 << 24) + 100, 128
    K, V = (torch.empty((1, 1, M, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.cat([torch.arange(7), torch.arange(M - 303, M)]).cuda()
    gen = torch.Generator(device="cuda").manual_seed(91)
    for t in (K, V):
        t[0, 0, rows] = torch.randn((len(rows), d), generator=gen, device="cuda").bfloat16()
    for n in (1, 3, 100):
        Q = normal((1, 4, n, d), "bf16", 92)
        O = grat.grat_window_attention_fwd(Q, K, V, 0.09, window=200, sinks=7)
        see = orc.window_seen(n, 310, 1, 200, 7, True)
        want, _, bO, _, _, _ = bounds(f64(Q), f64(K[:, :, rows]), f64(V[:, :, rows]), 0.09, see[:, None], "bf16")
        within(f64(O), want, bO, "O")


def test_streams_and_graphs():
    """A side stream, results allocated for it; a graph of a training step, replayed with new data between other work."""
    shape = (1, 4, 2, 700, 700, 100, 70, None, None, True)
    sets = [tensors(shape, "f16", 128, "heads", 100 + 10 * i) + (normal((1, 4, 700, 128), "f16", 105 + 10 * i),) for i in range(3)]

    def step(Q, K, V, dO, stream=None):
        O, lse = grat.grat_window_attention_fwd(Q, K, V, 0.1, window=100, sinks=70, return_lse=True, stream=stream)
        return (O, *grat.grat_window_attention_bwd(dO, Q, K, V, O, lse, 0.1, window=100, sinks=70, stream=stream))

    eager = [step(*t) for t in sets]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = step(*sets[0], stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, eager[0]))
    static = [t.clone() for t in sets[0]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*static)
    for i in (0, 1, 2, 1):
        for t, x in zip(static, sets[i]):
            t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, eager[i])), f"replay with data {i}"
        step(*sets[(i + 1) % 3])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("shape,pick", [
    ((4, 32, 32, 1100, 1100, 64, 70, [1100, 1100, 900, 66], None, True), [(0, 0), (2, 31), (3, 5)]),    # many tiles: two of first keys in parts beside others of one
    ((4, 64, 32, 1100, 1100, 64, 70, None, None, False), [(1, 17)]),                                    # ... both directions
    ((16, 32, 32, 300, 300, 40, 130, [300] * 15 + [131], None, True), [(0, 0), (9, 30), (15, 7)]),      # three tiles of first keys, as many as fill the chip: one part each
    ((1, 8, 1, 2500, 2500, 70, 600, None, None, True), None),                                           # few heads: first tiles in more parts than the others
])
def test_gradient_of_first_keys_in_parts(shape, pick, dtype, d):
    run_case(shape, dtype, d, where="tokens", backward=True, seed=111, pick=pick)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("shape,pick", [
    ((1, 8, 2, 60, 5000, 20, 700, [4990], None, True), None),                                           # 240 rows that see much the same first keys
    ((2, 8, 2, 64, 9000, 64, 6100, [9000, 40], [8700, -30], True), None),                               # ... in several parts; rows ahead of the first key
    ((2, 8, 2, 40, 3000, 25, 2000, None, [100, 2900], False), None),
    ((1, 8, 8, 2048, 4200, 100, 4000, None, None, True), [(0, 3)]),                                     # prompts that see more first keys than others
    ((4, 32, 32, 2700, 2700, 64, 2500, [2700, 2700, 2600, 900], None, True), [(0, 0), (3, 30)]),        # of 256 rows
])
def test_more_first_keys_than_others(shape, pick, dtype, d):
    run_case(shape, dtype, d, where="tokens", backward=True, seed=121, pick=pick)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("window,sinks", [(2 ** 31 - 1, 0), (2 ** 31 - 1, 2), (2 ** 31 - 2, 0), (None, 0), (1, 3)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [5, 70])
def test_positions_at_the_ends_of_their_type(n, causal, window, sinks, dtype, d):
    """The longest window is a limit all the same: it ends between the first keys for positions next to 2^31 and -2^31."""
    shape = (4, 4, 2, n, 140, window, sinks, [140, 140, 130, 140], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 30, -2 ** 31 + 69], causal)
    run_case(shape, dtype, d, where="tokens", backward=True, seed=131)
