"""The example: a layer that learns, and serves what the whole sequence gives."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.mark.parametrize("head_dim,q_heads,kv_heads", [(128, 8, 2), (64, 4, 4)])
def test_training_and_serving(head_dim, q_heads, kv_heads):
    import selected_attention
    # lists that hold every block: what is served then differs from the whole sequence by roundings only.  bf16 rounds Q, K, the
    # weights, O and the layer's result, 2^-8 each at most; five of them that agree in sign stay below 2^-5.
    losses, apart = selected_attention.main(n=500, top=8, q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim, steps=10, tokens=4)
    assert losses[-1] < 0.95 * losses[0]
    assert apart < 2.0 ** -5


def test_served_lists_are_their_own():
    import selected_attention
    losses, apart = selected_attention.main(n=1000, top=6, steps=3, tokens=3)
    assert losses[-1] < losses[0]
    assert apart < 1.0
