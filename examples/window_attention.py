"""One local attention layer: trained on whole sequences, then serving from caches in 8 bits, token by token or by trees of drafted tokens.

    python examples/window_attention.py

Training: Q, K, V are projected, turned by their positions, and every query attends the WINDOW newest tokens and the first SINKS ones; the gradient goes back
through attention and rotation.  Serving: the new tokens' K and V are kept in 8 bits, turned and rounded as they are written.  Drafted tokens, guesses
of how the sequence goes on, are written behind the committed ones as a tree and attended in one call, each along its own line; the rows of the line
that is accepted then move together (a draft's key is at the position of its depth, so it needs no turning).
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2505_14687_amd as grat

WINDOW, SINKS = 256, 4
LOCAL = dict(window=WINDOW, sinks=SINKS)


class Attend(torch.autograd.Function):
    """Q [B, Hq, N, d], K, V [B, Hkv, N, d], before rotation -> O [B, Hq, N, d]."""

    @staticmethod
    def forward(ctx, Q, K, V, table):
        Q, K = grat.grat_rotary(Q, K, table)
        O, lse = grat.grat_window_attention_fwd(Q, K, V, 1 / math.sqrt(Q.shape[3]), return_lse=True, **LOCAL)
        ctx.save_for_backward(Q, K, V, O, lse, table)
        return O

    @staticmethod
    def backward(ctx, dO):
        Q, K, V, O, lse, table = ctx.saved_tensors
        dQ, dK, dV = grat.grat_window_attention_bwd(dO, Q, K, V, O, lse, 1 / math.sqrt(Q.shape[3]), **LOCAL)
        grat.grat_rotary(dQ, dK, table, inverse=True, out=(dQ, dK))
        return dQ, dK, dV, None


class Layer(torch.nn.Module):
    def __init__(self, width, q_heads, kv_heads, head_dim, n_pos, dtype=torch.bfloat16):
        super().__init__()
        self.heads, self.head_dim = (q_heads, kv_heads, kv_heads), head_dim
        self.qkv = torch.nn.Linear(width, sum(self.heads) * head_dim, bias=False, dtype=dtype, device="cuda")
        self.out = torch.nn.Linear(q_heads * head_dim, width, bias=False, dtype=dtype, device="cuda")
        self.table = grat.grat_rotary_table(n_pos, [head_dim // 2])

    def project(self, x):   # views [B, H, N, d] of one buffer
        B, N, _ = x.shape
        return [t.transpose(1, 2) for t in self.qkv(x).view(B, N, sum(self.heads), self.head_dim).split(self.heads, dim=2)]

    def merge(self, O):
        return self.out(O.transpose(1, 2).flatten(2))

    def forward(self, x):
        return self.merge(Attend.apply(*self.project(x), self.table))


class Server:
    """Caches in 8 bits for `batch` sequences of up to n_max tokens, drafted ones included."""

    def __init__(self, layer, batch, n_max):
        self.layer, shape = layer, (batch, layer.heads[1], n_max, layer.head_dim)
        self.K, self.V = (torch.zeros(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        self.scales = {name: torch.zeros(shape[:3], device="cuda") for name in ("K_scale", "V_scale")}
        self.held = torch.zeros(batch, dtype=torch.int32, device="cuda")

    @torch.no_grad()
    def attend(self, x, parent=None, depth=None):
        """x [B, N, width] behind the committed tokens: the next ones, or drafted ones with their parents and depths [B, N]."""
        layer, N = self.layer, x.shape[1]
        positions = None if depth is None else (self.held[:, None] + depth).unsqueeze(-1).contiguous()
        Q, K, V = layer.project(x)
        Q = grat.grat_cache_append(Q, K, V, layer.table, self.K, self.V, self.held, positions=positions, **self.scales)
        O = grat.grat_cache_attention_fwd(Q, self.K, self.V, 1 / math.sqrt(layer.head_dim), k_len=self.held + N, parent=parent, **self.scales, **LOCAL)
        return layer.merge(O)

    def step(self, x):
        """The next tokens of every sequence, a prompt or a few."""
        y = self.attend(x)
        self.held += x.shape[1]
        return y

    def accept(self, line):
        """line [B, n] (int64): the drafted tokens that are accepted, from the first to the last of a line.  Their rows move together."""
        B, n = line.shape
        b, held = torch.arange(B, device="cuda")[:, None], self.held.long()[:, None]
        to, source = held + torch.arange(n, device="cuda"), held + line
        for t in (self.K.view(torch.uint8), self.V.view(torch.uint8), *self.scales.values()):
            t[b, :, to] = t[b, :, source]
        self.held += n


def main(batch=2, n=600, width=256, q_heads=8, kv_heads=2, head_dim=128, steps=20):
    """How far what is served is from the whole sequence, and what a tree of drafts gives from what serving its lines gives, relative to them."""
    torch.manual_seed(1)
    layer = Layer(width, q_heads, kv_heads, head_dim, n_pos=n + 16)
    x = torch.randn(batch, n, width, device="cuda").bfloat16()
    target = torch.randn(batch, 1, width, device="cuda").bfloat16().expand_as(x)
    optimizer = torch.optim.SGD(layer.parameters(), lr=2.0)
    for i in range(steps):
        loss = (layer(x) - target).float().square().mean()
        optimizer.zero_grad()
        loss.backward()
        optimizer.step()
        if i in (0, steps - 1):
            print(f"training: step {i + 1}, loss {float(loss.detach()):.4f}")

    with torch.no_grad():
        whole = layer(x)
    server, plain = Server(layer, batch, n + 16), Server(layer, batch, n + 16)
    served = [server.step(x[:, :n - 8])] + [server.step(x[:, i:i + 1]) for i in range(n - 8, n)]
    apart = float((torch.cat(served, 1) - whole).float().norm() / whole.float().norm())
    print(f"serving: a prompt of {n - 8} tokens and 8 more from caches in 8 bits, {apart:.4f} apart from the whole sequence")

    # two guesses at the next token, two more behind each, one of these goes on
    parent, depth = ([-1, -1, 0, 0, 1, 1, 4], [0, 0, 1, 1, 1, 1, 2])
    drafts = torch.randn(batch, len(parent), width, device="cuda").bfloat16()
    ints = lambda v: torch.tensor([v] * batch, dtype=torch.int32, device="cuda")   # noqa: E731
    y = server.attend(drafts, ints(parent), ints(depth))
    line = [1, 4, 6]
    server.accept(torch.tensor([line] * batch, device="cuda"))
    after = server.step(drafts[:, :1])
    plain.step(x)
    want = torch.cat([plain.step(drafts[:, t:t + 1]) for t in (*line, 0)], 1)
    drafted = float((torch.cat([y[:, line], after], 1) - want).float().norm() / want.float().norm())
    print(f"drafting: {len(line)} of {len(parent)} tokens accepted, {drafted:.4f} apart from serving them one by one")
    return apart, drafted


if __name__ == "__main__":
    main()
