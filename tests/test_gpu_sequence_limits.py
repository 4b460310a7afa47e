"""Token sequences at the ends of what is supported: caches beyond 4 GiB and element offsets beyond 2^31, lists of 2^18 keys."""
import math

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle as orc
from sequence_util import f64, normal
from test_gpu_sequence_attention import bounds, within

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24


def large(n, d, seed, rows):
    """[1, 1, n, d], of which only `rows` are filled."""
    t = torch.empty((1, 1, n, d), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t[0, 0, rows] = torch.randn((len(rows), d), generator=gen, device="cuda").bfloat16()
    return t


def test_means_beyond_4_gib():
    M, d, block = (1 << 24) + 100, 128, 32
    rows = torch.arange(M - 200, M, device="cuda")
    K = large(M, d, 600, rows)
    tail = f64(K[:, :, M - 200:])
    got = f64(grat.grat_block_means(K[:, :, M - 200:], block))      # a view that begins beyond 4 GiB
    want, size = orc.block_means(tail, block), orc.block_means(np.abs(tail), block)
    assert (np.abs(got - want) <= (block + 2) * EPS * size).all()
    # the whole cache, of which the blocks with the last 100 keys are looked at: only those are written
    blocks = -(-M // block)
    out = torch.full((1, 1, blocks, d), float("nan"), device="cuda")
    grat.grat_block_means(K, block, new=100, out=out)
    first = (M - 100) // block
    skip = first * block - (M - 200)
    want, size = orc.block_means(tail[:, :, skip:], block), orc.block_means(np.abs(tail[:, :, skip:]), block)
    assert torch.isnan(out[:, :, :first]).all()
    assert (np.abs(f64(out[:, :, first:]) - want) <= (block + 2) * EPS * size).all()


@pytest.mark.parametrize("N,share", [(1, 4), (70, 4)])     # 4 rows; 280 rows, whose parts are joined
def test_gradient_beyond_4_gib(N, share):
    """K, V, dK and dV of more than 4 GiB each; the lists' blocks lie at both ends and in between."""
    M, d, block = (1 << 24) + 100, 128, 64
    blocks = -(-M // block)
    chosen = [0, 5, blocks // 2, blocks - 2, blocks - 1]
    rows = torch.cat([torch.arange(j * block, min(M, (j + 1) * block)) for j in chosen]).cuda()
    K, V = large(M, d, 610, rows), large(M, d, 611, rows)
    Q, dO = normal((1, share, N, d), "bf16", 612), normal((1, share, N, d), "bf16", 613)
    count = torch.tensor([[[len(chosen)]]], dtype=torch.int32, device="cuda")
    index = torch.tensor([[[chosen]]], dtype=torch.int32, device="cuda")
    O, lse = grat.grat_selected_attention_fwd(Q, K, V, 0.09, count, index, q_group=N, block=block, return_lse=True)
    grads = [torch.empty_like(t) for t in (Q, K, V)]
    for t in grads[1:]:
        t.view(torch.int16).fill_(0x7fc0)                            # NaN: every row has to be written
    grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, 0.09, count, index, q_group=N, block=block, out=tuple(grads))
    at = rows.cpu().numpy()
    mask = (at[None, :] <= (M - N + np.arange(N))[:, None])[None, None]
    Ow, _, bO, _, want, lims = bounds(*(f64(t) for t in (Q, K[:, :, rows], V[:, :, rows])), 0.09, mask, "bf16", f64(dO))
    within(f64(O), Ow, bO, "O")
    for name, g, w, lim in zip(("dQ", "dK", "dV"), (grads[0], grads[1][:, :, rows], grads[2][:, :, rows]), want, lims):
        within(f64(g), w, lim, name)
    for t in grads[1:]:
        t[0, 0, rows] = 0
        bits = t.view(torch.int64).view(-1)                          # (four elements a number; no row of a block that is not listed has a gradient)
        assert not any(bool(part.any()) for part in bits.split(1 << 27))


@pytest.mark.parametrize("N,share,q_group,d,dtype", [
    (1, 4, 1, 128, "bf16"),       # one token, shared by workgroups
    (20, 4, 20, 128, "bf16"),     # 80 rows
    (20, 2, 20, 64, "f16"),       # 40 rows
    (260, 1, 1, 64, "bf16"),      # a workgroup a list
])
def test_lists_of_2_to_the_18_keys(N, share, q_group, d, dtype):
    M, block, top = 270000, 4096, 64
    blocks, groups = -(-M // block), -(-N // q_group)
    gen = np.random.default_rng(620)
    index = np.stack([gen.permutation(blocks)[:top] for _ in range(groups)])[None, None].astype(np.int32)
    count = np.full((1, 1, groups), top, np.int32)
    Q, dO = normal((1, share, N, d), dtype, 621), normal((1, share, N, d), dtype, 622)
    K, V = normal((1, 1, M, d), dtype, 623), normal((1, 1, M, d), dtype, 624)
    scale = 1 / math.sqrt(d)
    lists = torch.from_numpy(count).cuda(), torch.from_numpy(index).cuda()
    O, lse = grat.grat_selected_attention_fwd(Q, K, V, scale, *lists, q_group=q_group, block=block, return_lse=True)
    grads = grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, scale, *lists, q_group=q_group, block=block)
    mask = orc.attended(count, index, N, M, q_group, block, True)
    Ow, lw, bO, bl, want, lims = bounds(*(f64(t) for t in (Q, K, V)), scale, mask, dtype, f64(dO))
    within(f64(O), Ow, bO, "O")
    within(f64(lse), lw, bl, "lse")
    for name, g, w, lim in zip(("dQ", "dK", "dV"), grads, want, lims):
        within(f64(g), w, lim, name)
    with pytest.raises(grat.GratError):                              # one block more
        more = torch.zeros(1, 1, groups, top + 1, dtype=torch.int32, device="cuda")
        grat.grat_selected_attention_fwd(Q, K, V, scale, lists[0], more, q_group=q_group, block=block)
