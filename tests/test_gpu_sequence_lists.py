"""Block means, scores and the selection vs the float64 oracle.

Tolerances: a mean of n values is an fp32 sum of n terms, at most n * 2^-24 of the sum of their magnitudes off; a score is an fp32 dot
product of d terms with factors that are off by as much: (d + n + 4) * 2^-24 of the sum of the products' magnitudes.  Selection is exact."""
import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle as orc
from sequence_util import f64, ints, normal

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 128), ("f32", 64), ("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("B,H,M,block,lens,where", [
    (1, 1, 1, 32, None, "heads"),
    (2, 3, 129, 64, [129, 64], "tokens"),
    (3, 2, 300, 32, [0, 1, 299], "wide"),      # nothing valid; one key; a tail
    (1, 2, 1000, 256, [5000], "heads"),        # a length beyond the tensor is forced into it
    (2, 1, 4097, 4096, [-3, 4097], "heads"),
])
def test_means(dtype, d, B, H, M, block, lens, where):
    K = normal((B, H, M, d), dtype, 20, where)
    n = [min(max(l, 0), M) for l in lens] if lens else [M] * B
    for b in range(B):
        K[b, :, n[b]:] = float("nan")           # what is not valid is not read
    out = torch.full((B, H, -(-M // block), d), float("nan"), device="cuda")
    got = f64(grat.grat_block_means(K, block, k_len=ints(lens), out=out))
    want = orc.block_means(f64(K), block, lens)
    mag = orc.block_means(np.abs(f64(K)), block, lens)
    assert (np.abs(got - want) <= (min(block, M) + 2) * EPS * mag).all()


@pytest.mark.parametrize("new,M,block", [(1, 300, 32), (33, 300, 32), (300, 300, 64), (2, 65, 64)])
def test_means_of_new_keys(new, M, block):
    B, lens = 4, [M, 1, 0, min(M, 65)]
    K = normal((B, 2, M, 128), "bf16", 21)
    whole = grat.grat_block_means(K, block, k_len=ints(lens))
    kept = torch.full_like(whole, 7.0)
    grat.grat_block_means(K, block, k_len=ints(lens), new=new, out=kept)
    for b, n in enumerate(lens):
        lo, hi = max(0, n - new) // block, -(-n // block)
        assert torch.equal(kept[b, :, lo:hi], whole[b, :, lo:hi])
        assert bool((kept[b, :, :lo] == 7.0).all()) and bool((kept[b, :, hi:] == 7.0).all())


SHAPES = [  # B, Hq, Hkv, N, M, q_group, block, k_len, q_pos, causal
    (2, 4, 2, 1, 500, 1, 32, [500, 33], None, True),          # one token (few queries)
    (1, 8, 1, 5, 77, 1, 64, None, None, True),                # a few
    (3, 2, 2, 40, 40, 16, 32, [40, 7, 0], None, True),        # rows ahead of the first key, an empty sequence
    (1, 4, 4, 333, 333, 64, 64, None, None, True),            # the matrix product, odd sizes
    (1, 6, 2, 200, 3000, 1, 32, None, None, False),           # a list of its own for every query
    (2, 2, 1, 130, 260, 130, 32, [260, 100], [3, -60], True),  # positions that are given, one group
    (1, 16, 1, 70, 9000, 7, 32, [8999], None, True),
]


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f16", 64), ("f32", 64)])
@pytest.mark.parametrize("shape", SHAPES)
def test_scores(dtype, d, shape):
    B, Hq, Hkv, N, M, q_group, block, k_len, q_pos, causal = shape
    Q, K = normal((B, Hq, N, d), dtype, 22, "tokens"), normal((B, Hkv, M, d), dtype, 23)
    means = grat.grat_block_means(K, block, k_len=ints(k_len))
    out = torch.full((B, Hkv, -(-N // q_group), -(-M // block)), float("nan"), device="cuda")
    got = f64(grat.grat_block_scores(Q, means, 0.7, q_group, block, M, causal=causal, k_len=ints(k_len), q_pos=ints(q_pos), out=out))
    args = (q_group, block, M, causal, k_len, q_pos)
    want = orc.block_scores(f64(Q), f64(means), 0.7, *args)
    assert np.array_equal(np.isneginf(got), np.isneginf(want)) and not np.isnan(got).any()
    fin = np.isfinite(want)
    mag = orc.block_scores(np.abs(f64(Q)), np.abs(f64(means)), 0.7, *args)
    n = q_group * (Hq // Hkv)
    assert (np.abs(got[fin] - want[fin]) <= (d + n + 4) * EPS * mag[fin]).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("f32", 128)])
@pytest.mark.parametrize("share,q_group", [(1, 1), (3, 5), (2, 8), (16, 1), (1, 16), (17, 1)])
def test_scores_of_few_queries_a_group(dtype, d, share, q_group):
    """Mean queries of up to 16 rows, and one more; the last group is short."""
    N, M, block = 67 + 4 * q_group, 200, 32
    Q, K = normal((2, 2 * share, N, d), dtype, 26, "heads"), normal((2, 2, M, d), dtype, 27)
    means = grat.grat_block_means(K, block)
    got = f64(grat.grat_block_scores(Q, means, 0.3, q_group, block, M, causal=False))
    want = orc.block_scores(f64(Q), f64(means), 0.3, q_group, block, M, False)
    mag = orc.block_scores(np.abs(f64(Q)), np.abs(f64(means)), 0.3, q_group, block, M, False)
    assert (np.abs(got - want) <= (d + q_group * share + 4) * EPS * mag).all()


def expect_lists(scores, top, first, local, *where):
    want = orc.select_blocks(scores, top, first, local, *where)
    B, H, G = len(want), len(want[0]), len(want[0][0])
    count, index = np.zeros((B, H, G), np.int32), np.full((B, H, G, top), -1, np.int32)
    for b in range(B):
        for h in range(H):
            for g in range(G):
                count[b, h, g] = len(want[b][h][g])
                index[b, h, g, :count[b, h, g]] = want[b][h][g]
    return count, index


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "special"])
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("top,first,local", [(1, 0, 0), (4, 1, 2), (8, 0, 8), (40, 2, 3)])
def test_selection(kind, shape, top, first, local):
    B, Hq, Hkv, N, M, q_group, block, k_len, q_pos, causal = shape
    groups, blocks = -(-N // q_group), -(-M // block)
    gen = np.random.default_rng(24)
    scores = gen.standard_normal((B, Hkv, groups, blocks)).astype(np.float32)
    if kind == "ties":
        scores = np.round(2 * scores) / 2
    elif kind == "equal":
        scores[:] = -0.25
    elif kind == "special":
        pick = gen.integers(0, 8, scores.shape)
        for v, x in enumerate((np.nan, -np.inf, np.inf, 0.0, -0.0)):   # (the two zeros: see below)
            scores[pick == v] = x
        scores[pick == 4] = 0.0
        scores[pick == 5] = np.float32(-3.4e38)
    where = (N, M, q_group, block, causal, k_len, q_pos)
    count, index = grat.grat_select_blocks(torch.from_numpy(scores).cuda(), top, first, local, *where[:5], k_len=ints(k_len), q_pos=ints(q_pos))
    want_c, want_i = expect_lists(scores, top, first, local, *where)
    assert np.array_equal(count.cpu().numpy(), want_c)
    assert np.array_equal(index.cpu().numpy(), want_i)


def test_selection_orders_the_zeros_as_equal():
    scores = torch.tensor([[[[-0.0, 0.0, -0.0, 0.0]]]], device="cuda")
    _, index = grat.grat_select_blocks(scores, 2, 0, 0, n_q=1, n_k=128, q_group=1, block=32)
    assert index.flatten().tolist() == [0, 1]


@pytest.mark.parametrize("blocks", [64, 65, 128, 200, 256, 500, 512, 513, 2048, 2049, 8192, 8193, 20000, 32768])
def test_selection_of_every_length(blocks):
    """Every kind of launch, at its ends, with ties that cross the waves."""
    gen = np.random.default_rng(blocks)
    scores = np.round(8 * gen.standard_normal((1, 1, 3, blocks))).astype(np.float32)
    order = np.argsort(-scores[0, 0], axis=-1, kind="stable")
    for top in (1, 17, 300):
        _, index = grat.grat_select_blocks(torch.from_numpy(scores).cuda(), top, 0, 0, n_q=3, n_k=32 * blocks, q_group=1, block=32, causal=False)
        want = np.sort(order[:, :top], axis=-1)
        got = index.cpu().numpy()[0, 0][:, :want.shape[1]]
        assert np.array_equal(got, want)


@pytest.mark.parametrize("blocks", [1024, 1025, 1500, 2048, 4096, 4097, 16384, 16385])
@pytest.mark.parametrize("lists", [3, 1030])
def test_selection_of_few_and_many_lists(blocks, lists):
    if blocks > 2048 and lists > 3:
        lists = 40
    gen = np.random.default_rng(blocks + lists)
    scores = np.round(20 * gen.standard_normal((1, 1, lists, blocks))).astype(np.float32)
    order = np.argsort(-scores[0, 0], axis=-1, kind="stable")
    for top in (2, 29, 57, 300):
        count, index = grat.grat_select_blocks(torch.from_numpy(scores).cuda(), top, 0, 0, n_q=lists, n_k=32 * blocks, q_group=1, block=32, causal=False)
        assert (count == top).all()
        assert np.array_equal(index.cpu().numpy()[0, 0], np.sort(order[:, :top], axis=-1))
