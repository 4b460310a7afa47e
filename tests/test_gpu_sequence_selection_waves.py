"""Selection from 1 025 to 2 048 blocks, on both sides of every bound of the rule for the waves that share a list."""
import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", [1025, 2048])
@pytest.mark.parametrize("lists", [2047, 2048, 16383, 16384])
@pytest.mark.parametrize("top", [29, 30, 40, 41])
def test_selection(blocks, lists, top):
    gen = np.random.default_rng(blocks + lists + top)
    scores = np.round(20 * gen.standard_normal((1, 1, lists, blocks), dtype=np.float32))
    count, index = grat.grat_select_blocks(torch.from_numpy(scores).cuda(), top, 0, 0, n_q=lists, n_k=32 * blocks, q_group=1, block=32, causal=False)
    assert (count == top).all()
    pick = np.concatenate([np.arange(64), gen.integers(0, lists, 200), [lists - 1]])
    order = np.argsort(-scores[0, 0, pick], axis=-1, kind="stable")
    assert np.array_equal(index.cpu().numpy()[0, 0, pick], np.sort(order[:, :top], axis=-1))
