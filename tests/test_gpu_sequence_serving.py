"""What the example serves, step by step, vs the float64 oracle on the lists that each step selected; and which tokens a list depends on."""
import math
import os
import sys

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import sequence_oracle as orc
from sequence_util import f64, normal
from test_gpu_sequence_attention import bounds, within

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("head_dim,q_heads,kv_heads", [(128, 8, 2), (64, 4, 4)])
def test_every_step_attends_the_blocks_that_it_selected(monkeypatch, head_dim, q_heads, kv_heads):
    import selected_attention
    torch.manual_seed(3)
    batch, n, top, steps = 2, 700, 4, (500, 1, 1, 130, 1)            # a prompt, tokens, a chunk
    layer = selected_attention.Layer(256, q_heads, kv_heads, head_dim, top, n_pos=n)
    server = selected_attention.Server(layer, batch, n)
    seen = {}
    real = {name: getattr(grat, name) for name in ("grat_block_scores", "grat_select_blocks", "grat_selected_attention_fwd")}

    def record(name):
        def call(*args, **kw):
            r = real[name](*args, **kw)
            seen[name] = (args, kw, r)
            return r
        return call
    for name in real:
        monkeypatch.setattr(grat, name, record(name))
    x = torch.randn(batch, n, 256, device="cuda").bfloat16()
    with torch.no_grad():
        _, K, V = layer.project(x)
        held = 0
        for N in steps:
            server.step(x[:, held:held + N])
            held += N
            (Q, _, _, scale, count, index, q_group, block), kw, O = seen["grat_selected_attention_fwd"]
            Kr = grat.grat_rotary(Q.new_zeros(Q.shape[0], 1, held, head_dim), K[:, :, :held], layer.table)[1]
            assert torch.equal(server.K[:, :, :held], Kr) and torch.equal(server.V[:, :, :held], V[:, :, :held])
            means = orc.block_means(f64(Kr), block)
            mag = orc.block_means(np.abs(f64(Kr)), block)
            blocks = means.shape[2]
            assert (np.abs(f64(server.means)[:, :, :blocks] - means) <= (block + 2) * 2.0 ** -24 * mag).all()
            lens = [held] * batch
            local = min(top - 1, q_group // block + 1)
            scores = f64(seen["grat_block_scores"][2])
            want = orc.select_blocks(scores, top, 1, local, N, n, q_group, block, True, lens)
            for at in np.ndindex(*count.shape):
                assert index[at][:count[at]].tolist() == want[at[0]][at[1]][at[2]]
            mask = orc.attended(count.cpu().numpy(), index.cpu().numpy(), N, n, q_group, block, True, lens)
            assert mask.any(-1).all()
            Ow, _, bO, _, _, _ = bounds(f64(Q), f64(server.K), f64(server.V), scale, mask, "bf16")
            within(f64(O), Ow, bO, f"O after {held} tokens")


def lists_of(Q, K, q_group, block, top):
    N = Q.shape[2]
    scores = grat.grat_block_scores(Q, grat.grat_block_means(K, block), 1 / math.sqrt(Q.shape[3]), q_group, block, N)
    return grat.grat_select_blocks(scores, top, 1, 1, n_q=N, n_k=N, q_group=q_group, block=block)


def test_lists_of_single_queries_do_not_look_ahead():
    """q_group 1 and local 1: the newest block is in whatever its mean is, all others lie behind the query as a whole."""
    Q, K = normal((1, 4, 400, 64), "bf16", 630), normal((1, 2, 400, 64), "bf16", 631)
    count, index = lists_of(Q, K, 1, 32, 4)
    for n in (1, 31, 32, 33, 200, 399):
        c, i = lists_of(Q[:, :, :n], K[:, :, :n], 1, 32, 4)
        assert torch.equal(c, count[:, :, :n]) and torch.equal(i, index[:, :, :n])


def test_lists_of_groups_come_from_all_of_their_queries():
    """The list of a group changes with its last query, which the rows ahead of it share."""
    Q, K = normal((1, 1, 512, 64), "bf16", 632), normal((1, 1, 512, 64), "bf16", 633)
    _, index = lists_of(Q, K, 64, 32, 4)
    Q[:, :, -1] *= -64.0
    _, other = lists_of(Q, K, 64, 32, 4)
    assert torch.equal(index[:, :, :-1], other[:, :, :-1]) and not torch.equal(index[:, :, -1], other[:, :, -1])
