"""The example: its layer's gradients, and that serving, drafts included, gives what whole sequences give."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("head_dim,q_heads,kv_heads", [(128, 8, 2), (64, 4, 4)])
def test_it_runs(head_dim, q_heads, kv_heads):
    import window_attention
    apart, drafted = window_attention.main(n=400, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, steps=3)
    # served: K and V off by 2^-4 of themselves at most.  V's error stays that of O; a score's is below 2^-4 |q||k| scale, in which the weights'
    # largest relative error is e^x - 1: with scores of a trained layer that stay below 2 in size less than 2^-2, together below 0.3.
    assert apart < 0.3
    # the same rows either way, in other groupings of keys: bf16 rounds the weights, O and the layer's result, 2^-8 each at most
    assert drafted < 2.0 ** -6


@pytest.mark.parametrize("head_dim,q_heads,kv_heads", [(128, 4, 2), (64, 3, 3)])
def test_gradients(head_dim, q_heads, kv_heads):
    """Against autograd on elementary operations in fp32.  Q and K are rounded after rotation, and the weights, dS, O (in D) and the results, 2^-8 each at
    most: six that agree in sign stay below 2^-5 of a result's norm."""
    import window_attention as w
    torch.manual_seed(2)
    B, N = 2, 300
    Q, K, V, dO = (torch.randn(B, h, N, head_dim, device="cuda").bfloat16() for h in (q_heads, kv_heads, kv_heads, q_heads))
    table = w.grat.grat_rotary_table(N, [head_dim // 2])
    leaves = [t.clone().requires_grad_() for t in (Q, K, V)]
    O = w.Attend.apply(*leaves, table)
    O.backward(dO)

    def turn(x):
        c, s = table[:, :, 0], table[:, :, 1]
        a, b = x[..., :head_dim // 2], x[..., head_dim // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], -1)
    plain = [t.float().requires_grad_() for t in (Q, K, V)]
    share = q_heads // kv_heads
    k, v = turn(plain[1]).repeat_interleave(share, 1), plain[2].repeat_interleave(share, 1)
    i = torch.arange(N, device="cuda")
    see = (i <= i[:, None]) & ((i[:, None] - i < w.WINDOW) | (i < w.SINKS))
    s = (turn(plain[0]) @ k.transpose(2, 3).contiguous() / math.sqrt(head_dim)).masked_fill(~see, -math.inf)
    want = torch.softmax(s, -1) @ v
    want.backward(dO.float())
    for got, ref in [(O, want), *((a.grad, b.grad) for a, b in zip(leaves, plain))]:
        assert float((got.detach().float() - ref.detach()).norm()) <= 2.0 ** -5 * float(ref.detach().norm())
