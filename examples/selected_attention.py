"""One attention layer over selected key blocks: trained on whole sequences, then serving from a cache.

    python examples/selected_attention.py

Training: Q, K, V are projected, turned by their positions, key blocks are scored by their means, every group of 64 queries attends the blocks
selected for it, and the gradient goes back through attention and rotation (the selection is not differentiated).  Serving: a
prompt and then single tokens are appended to a cache, the means of the blocks that they touch are brought up to date, and each new token
attends the blocks that are selected for it alone.  The blocks of a group of 64 come from all of its queries, the later ones too, which a token
that is served alone has not got: where lists do not hold every block, what is served differs from the whole sequence by that choice.  A model
that has to be served as it was trained takes groups of one query (Q_GROUP = 1) throughout.
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_14687_amd as grat

BLOCK, Q_GROUP = 64, 64


def select(Q, means, scale, top, q_group, n_k, k_len=None):
    where = dict(q_group=q_group, block=BLOCK, k_len=k_len)
    scores = grat.grat_block_scores(Q, means, scale, n_k=n_k, **where)
    local = min(top - 1, q_group // BLOCK + 1)
    return grat.grat_select_blocks(scores, top, first=1, local=local, n_q=Q.shape[2], n_k=n_k, **where)


class Attend(torch.autograd.Function):
    """Q [B, Hq, N, d], K, V [B, Hkv, N, d], before rotation -> O [B, Hq, N, d]."""

    @staticmethod
    def forward(ctx, Q, K, V, table, top):
        scale = 1 / math.sqrt(Q.shape[3])
        Q, K = grat.grat_rotary(Q, K, table)
        count, index = select(Q, grat.grat_block_means(K, BLOCK), scale, top, Q_GROUP, K.shape[2])
        O, lse = grat.grat_selected_attention_fwd(Q, K, V, scale, count, index, Q_GROUP, BLOCK, return_lse=True)
        ctx.save_for_backward(Q, K, V, O, lse, count, index, table)
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, O, lse, count, index, table = ctx.saved_tensors
        dQ, dK, dV = grat.grat_selected_attention_bwd(dO, Q, K, V, O, lse, 1 / math.sqrt(Q.shape[3]), count, index, Q_GROUP, BLOCK)
        grat.grat_rotary(dQ, dK, table, inverse=True, out=(dQ, dK))
        return dQ, dK, dV, None, None


class Layer(torch.nn.Module):
    def __init__(self, width, q_heads, kv_heads, head_dim, top, n_pos, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.head_dim, self.top = (q_heads, kv_heads, kv_heads), head_dim, top
        self.qkv = torch.nn.Linear(width, sum(self.heads) * head_dim, bias=False, dtype=dtype, device="cuda")
        self.out = torch.nn.Linear(q_heads * head_dim, width, bias=False, dtype=dtype, device="cuda")
        self.table = grat.grat_rotary_table(n_pos, [head_dim // 2])

    def project(self, x):   # views [B, H, N, d] of one buffer
        B, N, _ = x.shape
        return [t.transpose(1, 2) for t in self.qkv(x).view(B, N, sum(self.heads), self.head_dim).split(self.heads, dim=2)]

    def merge(self, O):
        return self.out(O.transpose(1, 2).flatten(2))

    def forward(self, x):
        return self.merge(Attend.apply(*self.project(x), self.table, self.top))


class Server:
    """A cache for `batch` sequences of up to n_max tokens."""

    def __init__(self, layer, batch, n_max):
        self.layer, shape = layer, (batch, layer.heads[1], n_max, layer.head_dim)
        self.K, self.V = (torch.zeros(shape, dtype=layer.qkv.weight.dtype, device="cuda") for _ in range(2))
        self.means = torch.zeros((batch, layer.heads[1], -(-n_max // BLOCK), layer.head_dim), device="cuda")
        self.held = torch.zeros(batch, dtype=torch.int32, device="cuda")

    @torch.no_grad()
    def step(self, x):
        """x [B, N, width]: the next tokens of every sequence, a prompt or one each."""
        layer, scale, N = self.layer, 1 / math.sqrt(self.K.shape[3]), x.shape[1]
        q_group = 1 if N == 1 else Q_GROUP
        Q, K, V = layer.project(x)
        Q = grat.grat_rotary_append(Q, K, V, layer.table, self.K, self.V, start=self.held)
        self.held += N
        grat.grat_block_means(self.K, BLOCK, k_len=self.held, new=N, out=self.means)
        count, index = select(Q, self.means, scale, layer.top, q_group, self.K.shape[2], self.held)
        O = grat.grat_selected_attention_fwd(Q, self.K, self.V, scale, count, index, q_group, BLOCK, k_len=self.held)
        return layer.merge(O)


def train(layer, x, target, steps):
    optimizer = torch.optim.SGD(layer.parameters(), lr=2.0)
    losses = []
    for _ in range(steps):
        loss = (layer(x) - target).float().square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
    return losses


def main(batch=2, n=1000, width=256, q_heads=8, kv_heads=2, head_dim=128, top=8, steps=20, tokens=8):
    """Losses of the training steps, and how far what is served token by token is from the whole sequence, relative to it."""
    torch.manual_seed(1)
    layer = Layer(width, q_heads, kv_heads, head_dim, top, n_pos=n)
    x = torch.randn(batch, n, width, device="cuda").bfloat16()
    target = torch.randn(batch, 1, width, device="cuda").bfloat16().expand_as(x)
    losses = train(layer, x, target, steps)
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f}")

    whole = layer(x).detach()
    server = Server(layer, batch, n)
    served = [server.step(x[:, :n - tokens])] + [server.step(x[:, i:i + 1]) for i in range(n - tokens, n)]
    apart = float((torch.cat(served, 1) - whole)[:, -tokens:].float().norm() / whole[:, -tokens:].float().norm())
    print(f"serving: a prompt of {n - tokens} tokens and {tokens} more, {apart:.4f} apart from the whole sequence (lists of their own)")
    return losses, apart


if __name__ == "__main__":
    main()
