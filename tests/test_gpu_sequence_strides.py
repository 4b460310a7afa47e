"""Tensors whose strides are unusual, in both ways of marshalling: axes of one element, and inputs that repeat."""
import math

import pytest
import torch

import paper_2505_14687_amd as grat
from paper_2505_14687_amd import sequence as sq
from sequence_util import ints, normal


def odd(t):
    """The same tensor, with strides 3, 5 and 7 on its axes of one element."""
    return t.as_strided(t.shape, [k if n == 1 else s for n, s, k in zip(t.shape[:3], t.stride()[:3], (3, 5, 7))] + [1])


def test_strides_of_axes_of_one_element_do_not_count():
    t = odd(torch.zeros(1, 1, 1, 64))
    assert t.stride() == (3, 5, 7, 1)
    x = sq._tensor(t)
    assert (x.stride_b, x.stride_h, x.stride_n) == (0, 0, 64)
    x = sq._tensor(torch.zeros(2, 3, 4, 64))
    assert (x.stride_b, x.stride_h, x.stride_n) == (768, 256, 64)


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("B,H", [(1, 1), (1, 4), (3, 2)])
def test_axes_of_one_element(given, B, H):
    s = dict(stream=torch.cuda.current_stream() if given else None)
    Q, K, V, dO = (normal((B, H, 1, 128), "bf16", 500 + i) for i in range(4))
    table, start = grat.grat_rotary_table(10, [64]), ints([3] * B)
    lists = torch.ones(B, H, 1, dtype=torch.int32, device="cuda"), torch.zeros(B, H, 1, 1, dtype=torch.int32, device="cuda")

    def run(f):
        q, k, v, do = (f(t) for t in (Q, K, V, dO))
        cache = f(torch.zeros_like(K)), f(torch.zeros_like(K))
        qr, kr = grat.grat_rotary(q, k, table, start=start, out=(f(torch.empty_like(Q)), f(torch.empty_like(K))), **s)
        qa = grat.grat_rotary_append(q, k, v, table, *cache, ints([0] * B), **s)
        means = grat.grat_block_means(k, 32, **s)
        scores = grat.grat_block_scores(q, means, 0.1, 1, 32, 1, **s)
        O, lse = grat.grat_selected_attention_fwd(q, k, v, 0.1, *lists, 1, 32, return_lse=True, **s)
        return (qr, kr, qa, *cache, means, scores, O, lse, *grat.grat_selected_attention_bwd(do, q, k, v, f(O), lse, 0.1, *lists, 1, 32, **s))
    for x, y in zip(run(lambda t: t), run(odd)):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
def test_inputs_that_repeat(given):
    """One token's query for all sequences and heads, and one K/V head for several: views of stride 0."""
    s = dict(stream=torch.cuda.current_stream() if given else None)
    B, H, M, d = 3, 4, 100, 64
    q = normal((1, 1, 1, d), "f16", 510).expand(B, H, 1, d)
    k, v = (normal((B, 1, M, d), "f16", 511 + i).expand(B, H, M, d) for i in range(2))
    count = torch.full((B, H, 1), 2, dtype=torch.int32, device="cuda")
    index = torch.tensor([0, 2], dtype=torch.int32, device="cuda").repeat(B, H, 1, 1)
    scale = 1 / math.sqrt(d)

    def run(*t):
        O, lse = grat.grat_selected_attention_fwd(*t, scale, count, index, 1, 32, return_lse=True, **s)
        return (O, lse, *grat.grat_selected_attention_bwd(O, *t, O, lse, scale, count, index, 1, 32, **s))
    for x, y in zip(run(q, k, v), run(*(t.contiguous() for t in (q, k, v)))):
        assert torch.equal(x, y)
