"""Caches in 8 bits: rows written and read back, and attention of the newest tokens over caches of both kinds, vs the float64 oracle.

Rows: without rotation everything is exact (the scale is a power of two), so values and scales have to be the oracle's.  A turned number is off by 3 e of
|c x| + |s y| (two products and a sum in fp32, cos and sin rounded once; e = 2^-24), which may take it to the neighbouring e4m3 value where it is next to a border:
it is within its own rounding, 2^-4 of itself or 2^-10 s, of the number before rounding.
Attention: the bounds of test_gpu_sequence_attention.py on the values that the cache stands for; in 8 bits weights are rounded to bfloat16 (u = 2^-8), of half to
two such numbers (2^-17), and the scales cost two more fp32 roundings."""
import math

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle
from oracle import window_oracle as orc
from sequence_util import ROUND, TINY, TYPES, f64, ints, nan_like, normal
from test_gpu_sequence_attention import bounds, within

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
EIGHT = torch.float8_e4m3fn


def empty_cache(B, H, M, d, where="heads"):
    """Values and scales in which what nothing is written to stays NaN."""
    if where == "tokens":
        c = torch.full((B, M, H, d), 0x7f, dtype=torch.uint8, device="cuda").view(EIGHT).permute(0, 2, 1, 3)
        return c, torch.full((B, M, H), float("nan"), device="cuda").permute(0, 2, 1)
    if where == "wide":
        c = torch.full((B, H + 1, M + 2, d + 32), 0x7f, dtype=torch.uint8, device="cuda").view(EIGHT)[:, :H, 1:M + 1, 16:16 + d]
        return c, torch.full((B, H, 2, M + 3), float("nan"), device="cuda")[:, :, 1, 3:]
    return torch.full((B, H, M, d), 0x7f, dtype=torch.uint8, device="cuda").view(EIGHT), torch.full((B, H, M), float("nan"), device="cuda")


def odd_rows(x):
    """Zeros, infinities and NaN, the largest and the smallest numbers, borders of the scale and of the rounding."""
    info = torch.finfo(x.dtype)
    flat = x.view(-1, x.shape[-1])
    special = [torch.zeros(1), torch.tensor([float("nan"), 3.0]), torch.tensor([float("inf"), -float("inf"), 5.0]), torch.tensor([info.max, -1.0]),
               torch.tensor([info.tiny]), torch.tensor([info.tiny / 4]), torch.tensor([448.0, 1.0625, 1.1875, -17.0, 19.0]), torch.tensor([-449.0, 450.0]),
               torch.tensor([7.0, 0.013671875, 0.0009765625, 0.00048828125]), torch.tensor([float("nan")])]
    for i, values in enumerate(special[:len(flat)]):
        row = flat[i]
        if i in (0, 4, 5, 9):
            row.zero_()
        if i in (6, 7, 8):
            row.copy_(row.clamp(-1, 1))
        if i == 9:
            row.fill_(float("nan"))
        row[:len(values)] = values.to(x)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d,where", [(128, "tokens"), (64, "wide"), (64, "heads")])
def test_rows_are_the_oracles(dtype, d, where):
    B, H, N, M = 2, 3, 37, 50
    K, V = (normal((B, H, N, d), dtype, 200 + i, "heads") for i in range(2))
    odd_rows(K)
    odd_rows(V[1])
    (kc, ks), (vc, vs) = empty_cache(B, H, M, d, where), empty_cache(B, H, M, d, where)
    start = [20, -5]                                                  # the first sequence's last rows, the second's first are outside
    assert grat.grat_cache_append(None, K, V, None, kc, vc, ints(start), K_scale=ks, V_scale=vs) is None
    for x, c, s in ((K, kc, ks), (V, vc, vs)):
        values, scales = orc.quantise(f64(x), dtype == "f16")
        got, got_s = f64(c.float()), f64(s)
        want, want_s = np.full_like(got, np.nan), np.full_like(got_s, np.nan)
        for b in range(B):
            for i in range(N):
                if 0 <= start[b] + i < M:
                    want[b, :, start[b] + i], want_s[b, :, start[b] + i] = values[b, :, i], scales[b, :, i]
        assert np.array_equal(got_s, want_s, equal_nan=True)
        assert np.array_equal(got, want, equal_nan=True)
        k_len = [41, 0]
        for out_type in ("bf16", "f16", "f32"):
            back = grat.grat_cache_read(c, s, TYPES[out_type], k_len=ints(k_len))
            with np.errstate(over="ignore", invalid="ignore"):
                full = torch.from_numpy(got * got_s[..., None]).float().to(TYPES[out_type]).double().numpy()   # (e4m3 times a power of two: no double rounding)
            for b in range(B):
                full[b, :, k_len[b]:] = 0
            assert np.array_equal(f64(back), full, equal_nan=True)


def turned(x, cs, rot, layout):
    """Rows turned by cs [B, N, rot / 2, 2] in float64, and the sizes |c x| + |s y| that what fp32 loses goes by."""
    x, cs = f64(x), f64(cs)[:, None]
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if layout == "interleaved" else (slice(0, rot // 2), slice(rot // 2, rot))
    want, size = x.copy(), np.zeros_like(x)
    c, s = cs[..., 0], cs[..., 1]
    want[..., a], want[..., b] = c * x[..., a] - s * x[..., b], s * x[..., a] + c * x[..., b]
    size[..., a], size[..., b] = np.abs(c * x[..., a]) + np.abs(s * x[..., b]), np.abs(s * x[..., a]) + np.abs(c * x[..., b])
    return want, size


def is_turned(got, want, size, dtype):
    """Turned in fp32 (two products and a sum: 3 e of the size), rounded once."""
    assert (np.abs(f64(got) - want) <= ROUND[dtype] * np.abs(want) + 4 * EPS * size + TINY[dtype]).all()


@pytest.mark.parametrize("dtype,d,rot,layout", [("bf16", 128, 128, "half"), ("f16", 128, 64, "interleaved"), ("f32", 64, 64, "half"), ("f32", 128, 32, "interleaved"),
                                                ("f16", 64, 16, "half")])
@pytest.mark.parametrize("N,given", [(1, False), (45, False), (45, True)])
def test_turned_rows(dtype, d, rot, layout, N, given):
    B, Hq, H, M = 3, 6, 2, 100
    Q, K, V = normal((B, Hq, N, d), dtype, 210, "tokens"), normal((B, H, N, d), dtype, 211, "wide"), normal((B, H, N, d), dtype, 212)
    table = grat.grat_rotary_table(150, [rot // 2])
    start = [0, 17, 55]
    at = np.array(start)[:, None] + np.arange(N)
    positions = None
    if given:                                                         # positions of their own: rows are those of `start` all the same
        at = np.random.default_rng(5).integers(0, 150, (B, N))
        positions = ints(at)[..., None].contiguous()
    (kc, ks), (vc, vs) = empty_cache(B, H, M, d), empty_cache(B, H, M, d)
    Qt = grat.grat_cache_append(Q, K, V, table, kc, vc, ints(start), K_scale=ks, V_scale=vs, positions=positions, layout=layout)
    cs = table[torch.from_numpy(at).cuda()]
    is_turned(Qt, *turned(Q, cs, rot, layout), dtype)
    assert Qt.stride() == Q.stride()
    want, size = turned(K, cs, rot, layout)
    values, scales = orc.quantise(want)
    v_values, v_scales = orc.quantise(f64(V))
    for i in range(B):
        rows = slice(start[i], start[i] + N)
        assert np.array_equal(f64(ks[i, :, rows]), scales[i]) and np.array_equal(f64(vs[i, :, rows]), v_scales[i])
        assert np.array_equal(f64(vc[i, :, rows].float()), v_values[i])
        got = f64(kc[i, :, rows].float()) * scales[i][..., None]
        off = np.abs(got - want[i])
        assert (off <= 2.0 ** -4 * np.abs(want[i]) + 2.0 ** -10 * scales[i][..., None] + 4 * EPS * size[i]).all()
        assert (got != values[i] * scales[i][..., None]).mean() < 1e-3   # (a border is next to 2^-19 of all numbers)
    others = torch.ones((B, M), dtype=torch.bool)
    for i in range(B):
        others[i, start[i]:start[i] + N] = False
    assert ks.permute(0, 2, 1)[others].isnan().all() and vc.float().permute(0, 2, 1, 3)[others].isnan().all()


def test_caches_of_the_same_dtype():
    """Without scales: rows of the tensors' own type; Q in place; K and V alone."""
    B, Hq, H, N, M, d = 2, 4, 2, 9, 40, 128
    Q, K, V = normal((B, Hq, N, d), "bf16", 220), normal((B, H, N, d), "bf16", 221), normal((B, H, N, d), "bf16", 222)
    table, start = grat.grat_rotary_table(60, [64]), ints([3, 38])
    a = [torch.zeros((B, H, M, d), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    at = start[:, None].long() + torch.arange(N, device="cuda")
    want, size = turned(Q, table[at], d, "half")
    got = grat.grat_cache_append(Q, K, V, table, a[0], a[1], start)
    is_turned(got, want, size, "bf16")
    want, size = turned(K, table[at], d, "half")
    is_turned(a[0][0, :, 3:12], want[0], size[0], "bf16")
    is_turned(a[0][1, :, 38:], want[1, :, :2], size[1, :, :2], "bf16")
    assert torch.equal(a[1][0, :, 3:12], V[0]) and torch.equal(a[1][1, :, 38:], V[1, :, :2])
    assert not a[0][0, :, :3].any() and not a[0][0, :, 12:].any() and not a[1][1, :, :38].any()
    assert grat.grat_cache_append(None, K, V, table, a[2], a[3], start) is None
    assert all(torch.equal(a[i], a[i + 2]) for i in range(2))
    assert grat.grat_cache_append(Q, K, V, table, a[2], a[3], start, out=Q) is Q and torch.equal(Q, got)
    grat.grat_cache_append(None, K, V, None, a[2], a[3], start)
    assert torch.equal(a[2][0, :, 3:12], K[0]) and torch.equal(a[3][1, :, 38:], V[1, :, :2])


def test_positions_on_a_grid():
    B, H, N, d = 1, 2, 30, 64
    Q, K, V = (normal((B, H, N, d), "f16", 225 + i) for i in range(3))
    table = grat.grat_rotary_table(10, [10, 11, 11])
    at = torch.stack(torch.meshgrid(torch.arange(2), torch.arange(3), torch.arange(5), indexing="ij"), -1).view(1, 30, 3).int().cuda()
    kc, vc = (torch.zeros((B, H, 50, d), dtype=torch.float16, device="cuda") for _ in range(2))
    q = grat.grat_cache_append(Q, K, V, table, kc, vc, ints([7]), positions=at, axis_pairs=(10, 11, 11))
    axis = torch.tensor([0] * 10 + [1] * 11 + [2] * 11, device="cuda")
    cs = table[at[..., axis].long(), torch.arange(32, device="cuda")]
    is_turned(q, *turned(Q, cs, d, "half"), "f16")
    is_turned(kc[:, :, 7:37], *turned(K, cs, d, "half"), "f16")
    assert torch.equal(vc[:, :, 7:37], V)


# ---- attention ---------------------------------------------------------------------------------

# B, Hq, Hkv, N, M, window, sinks, k_len, tree
SHAPES = [
    (1, 4, 4, 1, 1, None, 0, None, False),                       # one key
    (3, 8, 2, 1, 700, 100, 5, [700, 1, 65], False),              # one token each
    (2, 16, 1, 1, 3000, 2000, 40, [2999, 130], False),           # keys shared by several workgroups
    (2, 40, 1, 1, 900, None, 0, [900, 0], False),                # 40 heads; an empty cache
    (2, 6, 2, 5, 400, 33, 32, None, False),                      # a few tokens: a chain
    (2, 8, 8, 3, 1500, None, 0, [1500, 2], False),               # rows ahead of the first key
    (1, 3, 1, 50, 333, 20, 1, [301], False),                     # 150 rows
    (2, 4, 2, 7, 90, None, 0, [90, 50], True),                   # trees
    (3, 8, 2, 13, 2000, 1900, 3, [2000, 13, 1500], True),        # 52 rows; nothing committed
    (2, 4, 1, 64, 1500, None, 0, [1500, 777], True),             # 256 rows
    (1, 2, 1, 256, 600, None, 0, [511], True),                   # the most drafted tokens
    (2, 4, 4, 40, 200, 6, 70, [200, 100], True),                 # a window shorter than the tree
    (2, 4, 2, 20, 64, 5, 3, [12, 25], True),                     # drafted tokens without a row; first keys among the drafted
    (1, 20, 1, 1, 5000, 4096, 4, None, True),                    # a tree of one token
    (2, 8, 2, 90, 700, 100, 3, [700, 311], False),               # 360 rows: a chain in the tiles of prompts
    (2, 12, 4, 60, 1800, 1500, 40, [1800, 59], True),            # 180 rows; a row without a key
    (1, 48, 2, 16, 1000, None, 0, [990], True),                  # 384 rows: two tiles
    (2, 4, 1, 64, 1500, 200, 3, [1500, 777], True),              # 256 rows that see different keys
    (2, 4, 1, 50, 900, 100, 5, [900, 333], False),               # 200 rows, a chain
    (2, 2, 1, 30, 700, 64, 2, [700, 100], False),                # 60 rows
    (2, 2, 1, 30, 700, 64, 2, [700, 100], True),
    (1, 1, 1, 256, 3000, 900, 2, [2900], True),                  # 256 rows in several parts
    (2, 1, 1, 250, 3000, 900, 2, [2900, 1300], False),           # ... of sequences of their own lengths
]


def parents(gen, B, N):
    """Parents near and far, several roots, and what is not a token ahead."""
    up = np.array([[int(gen.integers(max(-1, t - 6), t)) if t else -1 for t in range(N)] for _ in range(B)])
    if N > 6:
        up[:, N // 2] = -1
        up[0, 3], up[0, 4], up[-1, 5] = 3, N + 7, -9
    return up


def fill(x, see, eight):
    """A cache that holds x, NaN in the keys that no row sees; and what it stands for."""
    B, H, M, d = x.shape
    none = torch.from_numpy(~see.any(1)).to(x.device)[:, None].expand(B, H, M)
    if not eight:
        x[none] = float("nan")
        return x, None, x
    c, s = empty_cache(B, H, M, d, "tokens" if M % 2 else "wide")
    grat.grat_cache_append(None, x, x, None, c, c, ints([0] * B), K_scale=s, V_scale=s)
    c.view(torch.uint8)[none] = 0x7f
    s[none] = float("nan")
    return c, s, grat.grat_cache_read(c, s, torch.float32)


def run_case(shape, dtype, d, eight, seed=300, gain=1.0, up=None):
    B, Hq, Hkv, N, M, window, sinks, k_len, tree = shape
    gen = np.random.default_rng(seed)
    if tree and up is None:
        up = parents(gen, B, N)
    see = orc.tree_seen(up, M, window, sinks, k_len) if tree else orc.window_seen(N, M, B, window, sinks, True, k_len)
    Q = normal((B, Hq, N, d), dtype, seed, "tokens", gain)
    kc, ks, K = fill(normal((B, Hkv, M, d), dtype, seed + 1, "heads"), see, eight)
    vc, vs, V = fill(normal((B, Hkv, M, d), dtype, seed + 2, "heads"), see, eight)
    scale = 1.0 / math.sqrt(d)
    args = dict(k_len=ints(k_len), K_scale=ks, V_scale=vs, parent=ints(up) if tree else None, window=window, sinks=sinks)
    out = nan_like(Q)
    O, lse = grat.grat_cache_attention_fwd(Q, kc, vc, scale, return_lse=True, out=out, **args)
    assert O is out and torch.equal(O, grat.grat_cache_attention_fwd(Q, kc, vc, scale, **args))
    mask = np.repeat(see[:, None], Hkv, 1)
    with np.errstate(invalid="ignore"):
        Ow, lw, bO, bl, _, _ = bounds(f64(Q), f64(K), f64(V), scale, mask, dtype)
        if eight:
            PV = sequence_oracle.attention(f64(Q), f64(K), np.abs(f64(V)), scale, mask)[0]
            bO = bO + 8 * EPS * PV
    within(f64(O), Ow, bO, "O")
    got = f64(lse)
    assert np.array_equal(np.isneginf(got), np.isneginf(lw)), "rows that see nothing"
    fin = np.isfinite(lw)
    within(got[fin], lw[fin], bl[fin], "lse")


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(shape, dtype, d, eight):
    run_case(shape, dtype, d, eight)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,gain", [("bf16", 16.0), ("f16", 8.0)])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[6], SHAPES[9]])
def test_peaked_weights(shape, dtype, gain, eight):
    """Scores far apart: the reference maximum is refreshed on the way."""
    run_case(shape, dtype, 128, eight, seed=320, gain=gain)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,N,M,tree", [(64, 1, 2500, False), (65, 1, 2500, False), (7, 40, 3000, True), (2, 3, 20000, False), (1, 1, 30000, False),
                                        (3, 150, 2000, False)])
def test_lengths_of_their_own(B, N, M, tree, eight):
    """Sequences that share workgroups by their lengths: empty, short, as long as the cache; one more than share."""
    gen = np.random.default_rng(B + N)
    k_len = [int(n) for n in gen.integers(0, M + 1, B)]
    k_len[0], k_len[-1] = min(M, 777), 0 if B > 2 else M // 3
    run_case((B, 2, 1, N, M, None if N > 1 else 1800, 3 if N == 1 else 0, k_len, tree), "bf16", 64, eight, seed=360 + B)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("N,window,sinks,k_len", [(256, None, 0, 300), (256, 255, 0, 256), (256, 100, 0, 300), (256, 1, 0, 270), (256, 7, 30, 266), (200, 64, 250, 310),
                                                  (65, 63, 0, 80), (64, 64, 0, 64), (64, 3, 5, 61), (33, 32, 0, 33), (2, 1, 0, 9), (2, 1, 9, 9)])
def test_trees_of_long_lines(N, window, sinks, k_len, eight):
    """One line of N tokens, and one of two branches that leave it half way."""
    up = np.arange(N)[None].repeat(2, 0) - 1
    up[1, N // 2 + 1:] = np.maximum(np.arange(N // 2 + 1, N) - 2, N // 2)
    run_case((2, 2, 1, N, 320, window, sinks, [k_len, k_len], True), "bf16", 64, eight, seed=340, up=up)


@pytest.mark.parametrize("eight", [False, True])
def test_one_tree_for_all_sequences(eight):
    B, Hq, Hkv, N, M, d = 3, 4, 2, 9, 77, 64
    up = ints([-1, 0, 0, 1, 1, 2, 5, -1, 7])
    x = normal((B, Hkv, M, d), "bf16", 330)
    c, s = (x, None) if not eight else empty_cache(B, Hkv, M, d)
    if eight:
        grat.grat_cache_append(None, x, x, None, c, c, ints([0] * B), K_scale=s, V_scale=s)
    Q = normal((B, Hq, N, d), "bf16", 331)
    a = dict(K_scale=s, V_scale=s, k_len=ints([77, 60, 9]))
    want = grat.grat_cache_attention_fwd(Q, c, c, 0.1, parent=up.repeat(B, 1), **a)
    assert torch.equal(grat.grat_cache_attention_fwd(Q, c, c, 0.1, parent=up, **a), want)
    assert torch.equal(grat.grat_cache_attention_fwd(Q, c, c, 0.1, parent=up[None], **a), want)
    # a tree without branches is a chain (the keys may be taken in another order)
    line = np.arange(N)[None].repeat(B, 0) - 1
    see = orc.window_seen(N, M, B, 20, 2, True, [77, 60, 9])
    assert np.array_equal(see, orc.tree_seen(line, M, 20, 2, [77, 60, 9]))
    X = grat.grat_cache_read(c, s, torch.float32) if eight else x
    Ow, _, bO, _, _, _ = bounds(f64(Q), f64(X), f64(X), 0.1, np.repeat(see[:, None], Hkv, 1), "bf16")
    for up in (None, ints(line)):
        within(f64(grat.grat_cache_attention_fwd(Q, c, c, 0.1, parent=up, window=20, sinks=2, **a)), Ow, bO + 8 * EPS * np.abs(f64(X)).max(), "O")


@pytest.mark.parametrize("N", [70, 150])
@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_scales_of_any_value_and_many_rows(dtype, N):
    """140 rows: the scales stay beside the values.  300: what the cache stands for is rounded to the tensors' type first (half saturates)."""
    B, H, M, d = 1, 2, 500, 128
    gen = torch.Generator().manual_seed(337)
    c = [torch.randn((B, H, M, d), generator=gen).to(EIGHT).cuda() for _ in range(2)]
    s = [(0.1 + torch.rand((B, H, M), generator=gen)).cuda() for _ in range(2)]
    s[1][:, :, 3] = 3e4
    X = [x.float() * y[..., None] for x, y in zip(c, s)]
    if 2 * N > 256:
        X = [(x.clamp(-65504, 65504) if dtype == "f16" else x).to(TYPES[dtype]) for x in X]
    K, V = (f64(x) for x in X)
    Q = normal((B, 4, N, d), dtype, 338)
    O = grat.grat_cache_attention_fwd(Q, *c, 0.09, K_scale=s[0], V_scale=s[1])
    mask = np.repeat(orc.window_seen(N, M, B)[:, None], H, 1)
    Ow, _, bO, _, _, _ = bounds(f64(Q), K, V, 0.09, mask, dtype)
    if 2 * N <= 256:   # scales beside the values, as in run_case
        bO = bO + 8 * EPS * sequence_oracle.attention(f64(Q), K, np.abs(V), 0.09, mask)[0]
    within(f64(O), Ow, bO, "O")


def test_scales_of_any_value():
    """Scales that are not powers of two (calibrated ones), in reading and in attention."""
    B, H, M, d = 2, 2, 300, 128
    gen = torch.Generator().manual_seed(335)
    c = [torch.randn((B, H, M, d), generator=gen).to(EIGHT).cuda() for _ in range(2)]
    s = [(0.1 + torch.rand((B, H, M), generator=gen)).cuda() for _ in range(2)]
    K, V = (f64(x.float()) * f64(y)[..., None] for x, y in zip(c, s))
    back = grat.grat_cache_read(c[0], s[0], torch.float32)
    assert (np.abs(f64(back) - K) <= EPS * np.abs(K)).all()
    Q = normal((B, 4, 3, d), "f16", 336)
    O = grat.grat_cache_attention_fwd(Q, *c, 0.09, K_scale=s[0], V_scale=s[1])
    mask = np.repeat(orc.window_seen(3, M, B)[:, None], H, 1)
    Ow, _, bO, _, _, _ = bounds(f64(Q), K, V, 0.09, mask, "f16")
    bO += (2.0 ** -8 + 8 * EPS) * sequence_oracle.attention(f64(Q), K, np.abs(V), 0.09, mask)[0]
    within(f64(O), Ow, bO, "O")


def test_offsets_beyond_32_bits():
    """Caches in 8 bits whose rows lie beyond 4 GiB."""
    M, d = (1 << 25) + 100, 128
    c = [torch.empty((1, 1, M, d), dtype=torch.uint8, device="cuda").view(EIGHT) for _ in range(2)]
    s = [torch.empty((1, 1, M), device="cuda") for _ in range(2)]
    n = 303
    K, V = normal((1, 1, n, d), "bf16", 340), normal((1, 1, n, d), "bf16", 341)
    grat.grat_cache_append(None, K, V, None, *c, ints([M - n]), K_scale=s[0], V_scale=s[1])
    grat.grat_cache_append(None, K[:, :, :7], V[:, :, :7], None, *c, ints([0]), K_scale=s[0], V_scale=s[1])
    back = [grat.grat_cache_read(x[:, :, M - n:], y[:, :, M - n:], torch.float32) for x, y in zip(c, s)]
    rows = [torch.cat([x[:, :, :7], x], 2) for x in back]
    Q = normal((1, 4, 3, d), "bf16", 342)
    O = grat.grat_cache_attention_fwd(Q, *c, 0.09, K_scale=s[0], V_scale=s[1], window=200, sinks=7)
    mask = orc.window_seen(3, n + 7, 1, 200, 7)[:, None]
    Ow, _, bO, _, _, _ = bounds(f64(Q), f64(rows[0]), f64(rows[1]), 0.09, mask, "bf16")
    within(f64(O), Ow, bO + 8 * EPS * np.abs(Ow), "O")


def test_together_streams_and_graphs():
    """Steps of serving as a graph: drafted tokens turned and appended, attended as a tree, the cache read back."""
    B, Hq, Hkv, N, M, d = 2, 8, 2, 6, 900, 128
    table, up = grat.grat_rotary_table(1000, [64]), ints([[-1, 0, 0, 1, 3, -1], [-1, 0, 1, 2, 3, 4]])
    depth = ints([[0, 1, 1, 2, 3, 0], [0, 1, 2, 3, 4, 5]])
    start = ints([800, 333])
    sets = [[normal((B, h, N, d), "bf16", 350 + 10 * i + k) for k, h in enumerate((Hq, Hkv, Hkv))] for i in range(3)]
    old = [normal((B, Hkv, M, d), "bf16", 390 + i) for i in range(2)]
    fresh = []
    for x in old:
        c, s = empty_cache(B, Hkv, M, d)
        grat.grat_cache_append(None, x, x, None, c, c, ints([0, 0]), K_scale=s, V_scale=s)
        fresh.append((c, s))

    def step(Q, K, V, caches, stream=None):
        (kc, ks), (vc, vs) = caches
        q = grat.grat_cache_append(Q, K, V, table, kc, vc, start, K_scale=ks, V_scale=vs, positions=(start[:, None] + depth)[..., None].contiguous(), stream=stream)
        O = grat.grat_cache_attention_fwd(q, kc, vc, 0.09, k_len=start + N, K_scale=ks, V_scale=vs, parent=up, window=500, sinks=4, stream=stream)
        return O, grat.grat_cache_read(kc, ks, torch.float16, k_len=start + N, stream=stream)

    copies = lambda: [tuple(t.clone() for t in pair) for pair in fresh]   # noqa: E731
    eager = [step(*t, copies()) for t in sets]
    see = orc.tree_seen(up.cpu().numpy(), M, 500, 4, [806, 339])
    caches = copies()
    O, _ = step(*sets[0], caches)
    (kc, ks), (vc, vs) = copies()
    q = grat.grat_cache_append(*sets[0], table, kc, vc, start, K_scale=ks, V_scale=vs, positions=(start[:, None] + depth)[..., None].contiguous())
    K, V = (f64(grat.grat_cache_read(*pair, torch.float32)) for pair in caches)
    Ow, _, bO, _, _, _ = bounds(f64(q), K, V, 0.09, np.repeat(see[:, None], Hkv, 1), "bf16")
    within(f64(O), Ow, bO + 8 * EPS * np.abs(V).max(), "O")
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    mine = copies()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = step(*sets[0], mine)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, eager[0]))
    static, caches = [t.clone() for t in sets[0]], copies()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*static, caches)
    for i in (0, 1, 2, 1):
        for t, x in zip(static, sets[i]):
            t.copy_(x)
        for pair, was in zip(caches, fresh):
            for t, x in zip(pair, was):
                t.copy_(x)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(out, eager[i])), f"replay with data {i}"
        step(*sets[(i + 1) % 3], copies())


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("N,M,tree", [(1, 5000, False), (20, 3000, True), (150, 900, False)])
def test_a_graph_with_other_lengths(N, M, tree, eight):
    """Lengths and parents are read where they lie: a graph replays with others, as eager calls have them."""
    B, Hq, Hkv, d = 5, 4, 2, 64
    x = normal((B, Hkv, M, d), "bf16", 400)
    c, s = (x, None) if not eight else empty_cache(B, Hkv, M, d)
    if eight:
        grat.grat_cache_append(None, x, x, None, c, c, ints([0] * B), K_scale=s, V_scale=s)
    Q = normal((B, Hq, N, d), "bf16", 401)
    gen = np.random.default_rng(402)
    lengths = [ints([M] * B), ints([0, 1, N, M // 2, M]), ints([int(n) for n in gen.integers(0, M + 1, B)])]
    trees = [ints(parents(np.random.default_rng(403 + i), B, N)) if tree else None for i in range(3)]
    k_len, up = lengths[0].clone(), trees[0].clone() if tree else None

    def call(k, t):
        return grat.grat_cache_attention_fwd(Q, c, c, 0.125, k_len=k, K_scale=s, V_scale=s, parent=t, return_lse=True)

    eager = [call(k, t) for k, t in zip(lengths, trees)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(k_len, up)
    for i in (1, 0, 2, 1):
        k_len.copy_(lengths[i])
        if tree:
            up.copy_(trees[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[i])), f"replay with data {i}"
        call(lengths[(i + 1) % 3], trees[(i + 1) % 3])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("shape", [
    (2, 8, 2, 60, 5000, 20, 700, [4990, 611], False),                # 240 rows
    (1, 8, 2, 64, 9000, 64, 6100, [8000], True),                     # ... of a tree, in several parts
    (3, 6, 2, 40, 3000, 25, 2000, [3000, 30, 1999], True),           # first keys beyond the committed ones
])
def test_more_first_keys_than_others(shape, dtype, d, eight):
    run_case(shape, dtype, d, eight, seed=410)


@pytest.mark.parametrize("N", [3, 7, 20])
@pytest.mark.parametrize("d", [64, 128])
def test_scales_of_any_value_in_half_lose_nothing(N, d):
    """Few rows of half over 8 bits: a weight is two bfloat16 numbers, the second what the first leaves over, so that it is off by at most 2^-17 of itself (the rest
    is at most 2^-8, half a step of 2^-7 above 1, and rounded by half a step of 2^-16) in the place of the 2^-11 that `bounds` counts; scales that are no powers of two
    cost two fp32 roundings on the way, as in run_case.  (Weights of one bfloat16 number are 1.5 to 3.7 times beyond it.)"""
    B, H, M = 2, 2, 300
    gen = torch.Generator().manual_seed(431)
    c = [torch.randn((B, H, M, d), generator=gen).to(EIGHT).cuda() for _ in range(2)]
    s = [(0.1 + torch.rand((B, H, M), generator=gen)).cuda() for _ in range(2)]
    K, V = (f64(x.float()) * f64(y)[..., None] for x, y in zip(c, s))
    Q = normal((B, 4, N, d), "f16", 432)
    mask = np.repeat(orc.window_seen(N, M, B)[:, None], H, 1)
    Ow, _, bO, _, _, _ = bounds(f64(Q), K, V, 0.09, mask, "f16")
    PV = sequence_oracle.attention(f64(Q), K, np.abs(V), 0.09, mask)[0]
    O = grat.grat_cache_attention_fwd(Q, *c, 0.09, K_scale=s[0], V_scale=s[1])
    within(f64(O), Ow, bO + (2.0 ** -17 + 8 * EPS - ROUND["f16"]) * PV, "O")
