"""Attention within a window and over 8-bit caches, as measurable cases: what a model of local attention layers
trains on, and what serves it token by token or by trees of drafted tokens.

A case is one pass through one operator:

  "window"  attention of every token to its `window` newest positions and the first `sinks` tokens
  "train"   the same and its gradient
  "append"  serving: the new tokens' Q turned by their positions, their K turned and written into 8-bit caches with V
  "read"    an 8-bit cache back in the type that the other operators take
  "serve"   attention of the newest tokens over a cache in 8 or 16 bits: one token, a few, or a tree of drafted ones

q_heads / kv_heads query heads share a K/V head.  window 0: all positions.  Not causal: the window reaches as far
ahead as back.  Sequences of a batch that is "ragged" have lengths of their own (_lengths).  An 8-bit row is
float8_e4m3fn values times one power of two, the smallest with which the row's largest value is at most 448.

`own` chooses between the plain forms, written out in elementary operations, and the framework's kernels.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
EIGHT = torch.float8_e4m3fn


# ---------------------------------------------------------------------------------------------- cases

def _window(name, op, n_q, n_k, window, *, sinks=0, batch=1, q_heads=32, kv_heads=8, head_dim=128, causal=True, ragged=False,
            dtype="bf16", token_major=False):
    return {"name": name, "op": op, "n_q": n_q, "n_k": n_k, "window": window, "sinks": sinks, "batch": batch, "q_heads": q_heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "causal": causal, "ragged": ragged, "dtype": dtype, "token_major": token_major}


def _append(name, n_q, n_k, *, batch=1, q_heads=32, kv_heads=8, head_dim=128, rot=None, interleaved=False, tree=False, dtype="bf16",
            token_major=False):
    return {"name": name, "op": "append", "n_q": n_q, "n_k": n_k, "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot": rot or head_dim, "interleaved": interleaved, "tree": tree, "dtype": dtype,
            "token_major": token_major}


def _read(name, n_k, *, batch=1, kv_heads=8, head_dim=128, ragged=False, dtype="bf16"):
    return {"name": name, "op": "read", "n_k": n_k, "batch": batch, "kv_heads": kv_heads, "head_dim": head_dim, "ragged": ragged,
            "dtype": dtype}


def _serve(name, n_q, n_k, *, bits=8, tree=False, window=0, sinks=0, batch=1, q_heads=32, kv_heads=8, head_dim=128, ragged=False,
           dtype="bf16"):
    return {"name": name, "op": "serve", "n_q": n_q, "n_k": n_k, "bits": bits, "tree": tree, "window": window, "sinks": sinks,
            "batch": batch, "q_heads": q_heads, "kv_heads": kv_heads, "head_dim": head_dim, "causal": True, "ragged": ragged,
            "dtype": dtype}


def listed():
    return [
        # a prompt of 32768 tokens in one go, Q, K and V as the projections leave them
        _window("window_prompt", "window", 32768, 32768, 1024, sinks=4, token_major=True),
        # an encoder's layer: both directions, odd sizes, sequences of different lengths, small heads, three to a K/V head
        _window("window_both_f16", "window", 4001, 4001, 300, sinks=1, batch=3, q_heads=12, kv_heads=4, head_dim=64, causal=False,
                ragged=True, dtype="f16"),
        # a training step on 16384 tokens
        _window("train_long", "train", 16384, 16384, 1024, sinks=4),
        # a small training step: short odd sequences, small heads that share nothing, a short window
        _window("train_odd_f16", "train", 2047, 2047, 129, sinks=1, batch=2, q_heads=8, kv_heads=8, head_dim=64, dtype="f16"),
        # serving: one new token of each of 32 sequences, turned and appended
        _append("append_token", 1, 2048, batch=32),
        # a prompt's 8191 tokens written into the cache, half of the head turned
        _append("append_prompt_f16", 8191, 16384, batch=2, rot=64, interleaved=True, dtype="f16", token_major=True),
        # caches of 8 sequences of different lengths back in bf16, for a chunk of a prompt that follows
        _read("read_prompt", 16384, batch=8, ragged=True),
        # one short cache of small heads back in half
        _read("read_short_f16", 1000, kv_heads=4, head_dim=64, dtype="f16"),
        # the smallest serving call: one token, a window and the first tokens of a long cache, latency is all
        _serve("serve_token_window", 1, 131072, window=4096, sinks=4),
        # a full serving batch: 64 sequences of different lengths, all positions
        _serve("serve_tokens", 1, 8192, batch=64, ragged=True),
        # 64 drafted tokens of each of 4 sequences over their caches
        _serve("serve_tree", 64, 16384, batch=4, tree=True, ragged=True),
        # a few drafted tokens over a cache that stayed in half, eight heads to a K/V head
        _serve("serve_tree_f16", 13, 8000, bits=16, batch=4, q_heads=16, kv_heads=2, tree=True, window=2000, sinks=8, dtype="f16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = [work(c) for c in listed()]
    while True:
        case = _draw_any(rng)
        w = work(case)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most) and _scratch(case) <= 16e9:
            del case["name"]
            return case


def _draw_any(rng):
    op = rng.choice(["window", "window", "train", "train", "append", "read", "serve", "serve", "serve"])
    kv_heads, share = rng.choice([(8, 4), (8, 4), (4, 8), (2, 16), (8, 1), (4, 3), (1, 16), (3, 2)])
    heads = {"q_heads": kv_heads * share, "kv_heads": kv_heads, "head_dim": rng.choice([128, 128, 64])}
    dtype = rng.choice(["bf16", "bf16", "f16"] + (["f32"] if op in ("append", "read") else []))
    if op == "append":
        n_q = rng.choice([1, 1, _log_int(rng, 2, 64), _log_int(rng, 2, 8192)])
        return _append("", n_q, n_q + _log_int(rng, 16, 8192), batch=rng.choice([1, 2, 7, 16, 32]), rot=rng.choice([0, 0, heads["head_dim"] // 2]),
                       interleaved=rng.random() < 0.5, tree=n_q > 1 and n_q <= 64 and rng.random() < 0.6, dtype=dtype,
                       token_major=rng.random() < 0.4, **heads)
    if op == "read":
        batch = rng.choice([1, 1, 3, 8])
        del heads["q_heads"]
        return _read("", _log_int(rng, 1, 16384), batch=batch, ragged=batch > 1 and rng.random() < 0.5, dtype=dtype, **heads)
    window = rng.choice([0, _log_int(rng, 16, 4096), _log_int(rng, 16, 4096), _log_int(rng, 16, 4096)])
    sinks = rng.choice([0, 1, 4, _log_int(rng, 1, 128)]) if window else 0
    if op == "serve":
        batch = rng.choice([1, 1, 3, 8, 16, 64])
        n_q = rng.choice([1, 1, _log_int(rng, 2, 16), _log_int(rng, 2, 64)])
        return _serve("", n_q, n_q + _log_int(rng, 1, 131072 // (1 if batch < 8 else 8)), bits=rng.choice([8, 8, 16]),
                      tree=n_q > 1 and rng.random() < 0.7, window=window, sinks=sinks, batch=batch, ragged=batch > 1 and rng.random() < 0.6,
                      dtype=dtype, **heads)
    batch = rng.choice([1, 1, 2, 3])
    n_q = _log_int(rng, 5, 32768)
    n_k = n_q if op == "train" or rng.random() < 0.6 else n_q + _log_int(rng, 1, 16384)
    return _window("", op, n_q, n_k, window, sinks=sinks, batch=batch, causal=rng.random() < 0.75,
                   ragged=batch > 1 and rng.random() < 0.4, dtype=dtype, token_major=rng.random() < 0.4, **heads)


def _lengths(case):
    """Valid keys of every sequence of the batch."""
    n, batch = case["n_k"], case["batch"]
    return [max(1, n - (b * n) // (2 * batch)) if case.get("ragged") else n for b in range(batch)]


def _group(case):
    """Neighbouring queries that a plain form looks at together."""
    return case["n_q"] if case["op"] == "serve" else min(64, case["n_q"])


def _span(case):
    """Keys beside the first ones that a group of queries may see."""
    if not case["window"]:
        return case["n_k"]
    return min(case["n_k"], (case["window"] - 1) * (1 if case["causal"] else 2) + _group(case))


def _scratch(case):
    """Bytes of the largest intermediate of a plain form."""
    if case["op"] in ("append", "read"):
        return 0
    groups, keys = -(-case["n_q"] // _group(case)), _span(case) + case["sinks"]
    share = case["q_heads"] // case["kv_heads"]
    return 4 * case["batch"] * case["kv_heads"] * groups * keys * max(case["head_dim"], share * _group(case))


def _seen(case):
    """Of every sequence: (pairs of query row and key that a head has, different keys that some row sees)."""
    pairs, keys, n_q, window, sinks = 0, 0, case["n_q"], case["window"] or 1 << 40, case["sinks"]
    for length in _lengths(case):
        p = length - n_q + np.arange(n_q, dtype=np.int64)
        if case.get("tree"):   # the committed tokens and itself
            p = np.full(n_q, length - n_q, dtype=np.int64)
        hi = np.clip(p + 1 if case["causal"] else np.minimum(p + window, length), 0, length)
        lo = np.minimum(np.maximum(p - window + 1, 0), hi)
        first = np.minimum(sinks, hi if case["causal"] else length)
        pairs += int((hi - lo).sum() + np.clip(np.minimum(lo, first), 0, None).sum())
        low = int(lo[hi > lo].min()) if (hi > lo).any() else length
        keys += (n_q if case.get("tree") else 0) + (int(hi.max()) - low if (hi > lo).any() else 0) + min(int(first.max()), low)
    return pairs, min(keys, sum(_lengths(case)))


def work(case):
    es, d, batch = 4 if case["dtype"] == "f32" else 2, case["head_dim"], case["batch"]
    if case["op"] == "append":
        n, row = batch * case["n_q"], d + 4
        return {"bytes": n * (2 * case["q_heads"] * d * es + 2 * case["kv_heads"] * (d * es + row)),
                "flops": n * (3 * (case["q_heads"] + case["kv_heads"]) * case["rot"] + 4 * case["kv_heads"] * d)}
    if case["op"] == "read":
        rows = case["kv_heads"] * sum(_lengths(case))
        return {"bytes": rows * (d + 4) + batch * case["kv_heads"] * case["n_k"] * d * es, "flops": rows * d}
    pairs, keys = _seen(case)
    q, row = batch * case["q_heads"] * case["n_q"] * d * es, (d + 4 if case.get("bits") == 8 else d * es)
    kv = 2 * case["kv_heads"] * keys * row
    if case["op"] == "train":
        return {"bytes": 4 * q + 2 * kv, "flops": 14 * d * pairs * case["q_heads"]}
    return {"bytes": 2 * q + kv, "flops": 4 * d * pairs * case["q_heads"]}


# --------------------------------------------------------------------------------------------- inputs

def _quantise(x):
    """Rows of x in 32 (or 64) bits -> float8_e4m3fn values and the rows' powers of two.  (448 = 7/8 2^9.)"""
    most, power = torch.frexp(x.abs().amax(-1))
    power = torch.where(most > 0, power + torch.where(most > 0.875, -8, -9), 0)
    return torch.ldexp(x, -power[..., None]).to(EIGHT), torch.ldexp(torch.ones_like(most), power)


def _frequencies(case):
    """Radians per position in 64 bits of every turned pair."""
    pairs = case["rot"] // 2
    return torch.tensor([10000.0 ** (-i / pairs) for i in range(pairs)], dtype=torch.float64, device="cuda")


def prepare(case, seed):
    dtype, B, Hkv, d = DTYPES[case["dtype"]], case["batch"], case["kv_heads"], case["head_dim"]
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(heads, n):
        if case.get("token_major"):
            return torch.randn((B, n, heads, d), generator=gen, device="cuda", dtype=dtype).permute(0, 2, 1, 3)
        return torch.randn((B, heads, n, d), generator=gen, device="cuda", dtype=dtype)

    def ints(values):
        return torch.tensor(values, dtype=torch.int32, device="cuda")

    def cache():   # as earlier tokens have left it
        rows = torch.randn((B, Hkv, case["n_k"], d), generator=gen, device="cuda", dtype=torch.bfloat16)
        return _quantise(rows.float())

    state = {"case": case, "scale": 1.0 / math.sqrt(d)}
    if case.get("ragged"):
        state["k_len"] = ints(_lengths(case))
    if case.get("tree"):   # every drafted token goes on from one of the eight ahead of it, or from the newest committed one
        t = torch.arange(case["n_q"], device="cuda")
        back = (torch.rand((B, case["n_q"]), generator=gen, device="cuda") * t.clamp(max=8)).long()
        state["parent"] = (t - 1 - back).clamp(min=-1).int()
    if case["op"] in ("window", "train"):
        state["q"], state["k"], state["v"] = normal(case["q_heads"], case["n_q"]), normal(Hkv, case["n_k"]), normal(Hkv, case["n_k"])
        if case["op"] == "train":
            state["do"] = normal(case["q_heads"], case["n_q"])
    elif case["op"] == "append":
        n = case["n_q"]
        state["q"], state["k"], state["v"] = normal(case["q_heads"], n), normal(Hkv, n), normal(Hkv, n)
        start = ints([max(0, case["n_k"] - n - 3 * b) for b in range(B)])   # tokens already in each cache
        state["start"] = start
        (state["k_cache"], state["k_scale"]), (state["v_cache"], state["v_scale"]) = cache(), cache()
        if case["tree"]:   # a drafted token's position follows from its place in the tree, its row does not
            state["positions"] = (start[:, None] + _reach(state["parent"]).sum(-1).int() - 1)[..., None].contiguous()
        angle = torch.arange(case["n_k"], dtype=torch.float64, device="cuda")[:, None] * _frequencies(case)
        state["table"] = torch.stack([angle.cos(), angle.sin()], -1).float()   # kept beside the weights
    elif case["op"] == "read":
        state["k_cache"], state["k_scale"] = cache()
    else:
        state["q"] = normal(case["q_heads"], case["n_q"])
        if case["bits"] == 8:
            (state["k_cache"], state["k_scale"]), (state["v_cache"], state["v_scale"]) = cache(), cache()
        else:
            state["k_cache"], state["v_cache"] = normal(Hkv, case["n_k"]), normal(Hkv, case["n_k"])
    return state


# ---------------------------------------------------------------------------------------- plain forms

def _reach(parent):
    """[B, n, n]: 1 where token a is t's ancestor or t itself.  (I + P + P^2 + ... = (I - P)^-1, P of parents.)"""
    n = parent.shape[1]
    t = torch.arange(n, device="cuda")
    step = (parent.long()[..., None] == t).float()
    eye = torch.eye(n, device="cuda").expand_as(step).contiguous()
    return torch.linalg.solve_triangular(eye - step, eye, upper=False, unitriangular=True)


def _plain_read(state):
    case, n = state["case"], state["case"]["n_k"]
    rows = state["k_cache"].float() * state["k_scale"][..., None]
    if "k_len" in state:
        there = torch.arange(n, device="cuda") < state["k_len"][:, None].long()
        rows = torch.where(there[:, None, :, None], rows, torch.zeros((), device="cuda"))
    return rows.to(DTYPES[case["dtype"]])


def _plain_turn(case, x, cos, sin):
    """x [B, H, N, d] in 32 bits turned by cos, sin [B, 1, N, pairs]; dims behind the turned ones pass through."""
    rot, x = case["rot"], x.float()
    if case["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(state):
    case, n = state["case"], state["case"]["n_q"]
    rows = state["start"].long()[:, None] + torch.arange(n, device="cuda")                      # [B, n]
    at = state["positions"][..., 0].long() if "positions" in state else rows
    cos, sin = state["table"][at].unsqueeze(1).unbind(-1)
    q, k = _plain_turn(case, state["q"], cos, sin).to(state["q"].dtype), _plain_turn(case, state["k"], cos, sin)
    where = (torch.arange(case["batch"], device="cuda")[:, None, None], torch.arange(case["kv_heads"], device="cuda")[None, :, None],
             rows[:, None])
    k8, k_scale = _quantise(k)
    v8, v_scale = _quantise(state["v"].float())
    state["k_cache"].view(torch.uint8)[where] = k8.view(torch.uint8)
    state["v_cache"].view(torch.uint8)[where] = v8.view(torch.uint8)
    state["k_scale"][where] = k_scale
    state["v_scale"][where] = v_scale
    return q, state["k_cache"], state["v_cache"], state["k_scale"], state["v_scale"]


def _length(state):
    case = state["case"]
    if "k_len" in state:
        return state["k_len"].long()
    return torch.full((case["batch"],), case["n_k"], dtype=torch.long, device="cuda")


def _gather(state, name, at):
    """Rows `at` [B, groups, keys] of K or V in 32 bits: [B, Hkv, groups, keys, d]."""
    case = state["case"]
    where = (torch.arange(case["batch"], device="cuda")[:, None, None, None],
             torch.arange(case["kv_heads"], device="cuda")[None, :, None, None], at[:, None])
    x = state[name + "_cache"] if name + "_cache" in state else state[name]
    if x.dtype == EIGHT:
        return x.view(torch.uint8)[where].view(EIGHT).float() * state[name + "_scale"][where][..., None]
    return x[where].float()


def _rows(case, x):
    """[B, Hq, n_q, d] -> [B, Hkv, groups, share * group, d] in 32 bits; rows behind the last query are 0."""
    B, Hkv, share, d, group = case["batch"], case["kv_heads"], case["q_heads"] // case["kv_heads"], x.shape[-1], _group(case)
    groups = -(-case["n_q"] // group)
    x = torch.nn.functional.pad(x.float(), (0, 0, 0, groups * group - case["n_q"]))
    return x.view(B, Hkv, share, groups, group, d).transpose(2, 3).flatten(3, 4)


def _unrows(case, x):
    B, Hkv, share, d, group = case["batch"], case["kv_heads"], case["q_heads"] // case["kv_heads"], x.shape[-1], _group(case)
    x = x.view(B, Hkv, -1, share, group, d).transpose(2, 3)
    return x.reshape(B, Hkv * share, -1, d)[:, :, :case["n_q"]]


def _keys(state):
    """Keys that the groups look at, [B, groups, keys], and which of them every row sees, [B, groups, group, keys]."""
    case, length = state["case"], _length(state)
    group, n_k, sinks, span = _group(case), case["n_k"], min(case["sinks"], case["n_k"]), _span(case)
    groups, window = -(-case["n_q"] // group), case["window"] or 1 << 40
    t = torch.arange(groups * group, device="cuda")
    there = (t < case["n_q"]).view(1, groups, group, 1)
    base = length - case["n_q"]
    first = (base[:, None] + t[::group] - window + 1).clamp(min=0)                              # of a group's window
    near = torch.minimum(first, torch.full_like(first, n_k - span))[..., None] + torch.arange(span, device="cuda")
    at = torch.cat([torch.arange(sinks, device="cuda").expand(near.shape[0], groups, sinks), near], -1)
    once = torch.cat([torch.ones_like(at[..., :sinks], dtype=torch.bool), near >= sinks], -1)   # (no key twice)
    key = at[:, :, None]
    valid = there & once[:, :, None] & (key < length.view(-1, 1, 1, 1))
    if not case.get("tree"):
        p = (base[:, None] + t).view(-1, groups, group, 1)
        if case["causal"]:
            return at, valid & (key <= p) & ((p - key < window) | (key < sinks))
        return at, valid & (((p - key).abs() < window) | (key < sinks))
    reach = _reach(state["parent"])
    depth = reach.sum(-1).long() - 1
    j = key - base.view(-1, 1, 1, 1)                                                            # < 0: committed
    drafted = j.clamp(0, case["n_q"] - 1).expand(-1, 1, group, -1)[:, 0]
    p = (base[:, None] + depth).view(-1, 1, group, 1)
    own_p = (base[:, None, None] + torch.gather(depth[:, None].expand(-1, group, -1), 2, drafted))[:, None]
    p_key = torch.where(j < 0, key, own_p)
    line = (j < 0) | (torch.gather(reach, 2, drafted)[:, None] > 0)
    return at, valid & line & ((p - p_key < window) | (p_key < sinks))


def _plain_attend(state):
    case = state["case"]
    at, sees = _keys(state)
    q, k, v = _rows(case, state["q"]), _gather(state, "k", at), _gather(state, "v", at)
    share, group = case["q_heads"] // case["kv_heads"], _group(case)
    s = (q @ k.transpose(3, 4)) * state["scale"]
    shape = s.shape
    s = torch.where(sees[:, None, :, None], s.view(*shape[:3], share, group, shape[4]), torch.full((), -math.inf, device="cuda")).view(shape)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, torch.zeros((), device="cuda"), m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total == 0, torch.ones((), device="cuda"), total)
    return q, k, v, p, p @ v, at


def _plain_train(state):
    case, dtype, d = state["case"], state["q"].dtype, state["case"]["head_dim"]
    q, k, v, p, o, at = _plain_attend(state)
    do = _rows(case, state["do"])
    ds = p * (do @ v.transpose(3, 4) - (do * o).sum(-1, keepdim=True)) * state["scale"]
    dq = ds @ k
    heads, n = case["batch"] * case["kv_heads"], case["n_k"]
    to = (at[:, None] + (torch.arange(heads, device="cuda") * n).view(case["batch"], case["kv_heads"], 1, 1)).flatten()
    dk, dv = (torch.zeros((heads * n, d), device="cuda") for _ in range(2))
    dk.index_add_(0, to, (ds.transpose(3, 4) @ q).view(-1, d))
    dv.index_add_(0, to, (p.transpose(3, 4) @ do).view(-1, d))
    return (_unrows(case, o).to(dtype), _unrows(case, dq).to(dtype), dk.view(state["k"].shape).to(dtype), dv.view(state["v"].shape).to(dtype))


def _plain(state):
    op = state["case"]["op"]
    if op == "append":
        return _plain_append(state)
    if op == "read":
        return _plain_read(state)
    if op == "train":
        return _plain_train(state)
    return _unrows(state["case"], _plain_attend(state)[4]).to(state["q"].dtype)


# ------------------------------------------------------------------------------------ the framework's

def _own(state):
    import paper_2505_14687_amd as grat
    case, op = state["case"], state["case"]["op"]
    if op == "append":
        q = grat.grat_cache_append(state["q"], state["k"], state["v"], state["table"], state["k_cache"], state["v_cache"], state["start"],
                                   K_scale=state["k_scale"], V_scale=state["v_scale"], positions=state.get("positions"),
                                   layout="interleaved" if case["interleaved"] else "half")
        return q, state["k_cache"], state["v_cache"], state["k_scale"], state["v_scale"]
    if op == "read":
        return grat.grat_cache_read(state["k_cache"], state["k_scale"], DTYPES[case["dtype"]], k_len=state.get("k_len"))
    where = {"window": case["window"] or None, "sinks": case["sinks"], "k_len": state.get("k_len")}
    if op == "serve":
        return grat.grat_cache_attention_fwd(state["q"], state["k_cache"], state["v_cache"], state["scale"], K_scale=state.get("k_scale"),
                                             V_scale=state.get("v_scale"), parent=state.get("parent"), **where)
    where["causal"] = case["causal"]
    if op == "window":
        return grat.grat_window_attention_fwd(state["q"], state["k"], state["v"], state["scale"], **where)
    o, lse = grat.grat_window_attention_fwd(state["q"], state["k"], state["v"], state["scale"], return_lse=True, **where)
    grads = grat.grat_window_attention_bwd(state["do"], state["q"], state["k"], state["v"], o, lse, state["scale"], **where)
    return (o, *grads)


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------- in 64 bits

def _exact_turn(case, x, angle):
    """Every turned pair as a complex number times e^(i angle)."""
    rot, x = case["rot"], x.double()
    out = x.clone()
    a, b = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., a], x[..., b]) * torch.polar(torch.ones_like(angle), angle)
    out[..., a], out[..., b] = z.real, z.imag
    return out


def _exact_append(case, state):
    n, start = case["n_q"], state["start"].tolist()
    rows = torch.stack([torch.arange(s, s + n, device="cuda") for s in start])
    at = state["positions"][..., 0] if "positions" in state else rows
    angle = (at.double()[..., None] * _frequencies(case))[:, None]
    out = [_exact_turn(case, state["q"], angle)]
    caches, scales = [], []
    for name, x in (("k", _exact_turn(case, state["k"], angle)), ("v", state["v"].double())):
        values, scale = state[name + "_cache"].double(), state[name + "_scale"].double()
        most = x.abs().amax(-1)
        power = torch.where(most > 0, torch.ceil(torch.log2(most.clamp(min=1e-300) / 448)), 0)
        for b, s in enumerate(start):
            values[b, :, s:s + n] = (x[b] * 2.0 ** -power[b][..., None]).to(EIGHT).double()
            scale[b, :, s:s + n] = 2.0 ** power[b]
        caches.append(values)
        scales.append(scale)
    return (*out, *caches, *scales)


def _exact_mask(case, length, rows, keys, parent):
    """Whether the query in row r sees key j, for every r of `rows` and j of `keys`."""
    window, base = case["window"] or 1 << 40, length - case["n_q"]
    if parent is None:
        p, q = (rows + base)[:, None], keys[None]
        near = (q <= p) & (q > p - window) if case["causal"] else (q < p + window) & (q > p - window)
        return (keys < length) & (near | ((q < case["sinks"]) & ((q <= p) if case["causal"] else (q >= 0))))
    lines, depth = [], []
    for t, up in enumerate(parent):   # each token's line of ancestors
        lines.append(lines[up] + [t] if up >= 0 else [t])
        depth.append(len(lines[t]) - 1)
    mask = torch.zeros((len(parent), case["n_k"]), dtype=torch.bool)
    for t, line in enumerate(lines):
        p = base + depth[t]
        mask[t, max(0, p - window + 1):max(0, base)] = True
        mask[t, :max(0, min(case["sinks"], base))] = True
        for a in line:
            if base + a >= 0 and (depth[t] - depth[a] < window or base + depth[a] < case["sinks"]):
                mask[t, base + a] = True
    return mask.cuda()[rows][:, keys]


def exact(case, seed):
    state = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, state)
    if case["op"] == "read":
        x = state["k_cache"].double() * state["k_scale"].double()[..., None]
        for b, length in enumerate(_lengths(case)):
            x[b, :, length:] = 0
        return x
    Hkv, share, d, n_q, train = case["kv_heads"], case["q_heads"] // case["kv_heads"], case["head_dim"], case["n_q"], case["op"] == "train"
    names = ("q", "q", "k", "v") if train else ("q",)
    want = [torch.zeros(state[t].shape, dtype=torch.float64, device="cuda") for t in names]
    for b, length in enumerate(_lengths(case)):
        k, v = (state[t + "_cache" if case["op"] == "serve" else t][b].double() for t in ("k", "v"))
        if case.get("bits") == 8:
            k, v = k * state["k_scale"][b].double()[..., None], v * state["v_scale"][b].double()[..., None]
        step = n_q if case.get("tree") else min(512, max(1, (1 << 26) // (case["q_heads"] * min(case["n_k"], 2 * _span(case)))))
        for lo in range(0, n_q, step):   # a slice of queries and the keys around it
            rows = torch.arange(lo, min(n_q, lo + step), device="cuda")
            first, last = 0, length
            if case["window"]:
                first = min(length, max(0, lo + length - n_q - case["window"] + 1, case["sinks"]))
                last = length if case.get("tree") else max(first, min(length, int(rows[-1]) + length - n_q + case["window"]))
            keys = torch.cat([torch.arange(min(first, case["sinks"], length), device="cuda"), torch.arange(first, last, device="cuda")])
            if case["window"] and first < case["sinks"]:
                keys = torch.arange(max(last, min(length, case["sinks"])), device="cuda")
            if not len(keys):
                continue
            mask = _exact_mask(case, length, rows, keys, state["parent"][b].tolist() if case.get("tree") else None)
            q = state["q"][b, :, rows].double().view(Hkv, share, len(rows), d)
            s = (q.flatten(1, 2) @ k[:, keys].transpose(1, 2) * state["scale"]).view(Hkv, share, len(rows), -1)
            p = torch.softmax(s.masked_fill_(~mask, -math.inf), -1).nan_to_num_(0.0).flatten(1, 2)
            o = p @ v[:, keys]
            want[0][b, :, rows] = o.view(-1, len(rows), d)
            if train:
                do = state["do"][b, :, rows].double().view(Hkv, -1, d)
                ds = p * (do @ v[:, keys].transpose(1, 2) - (do * o).sum(-1, keepdim=True)) * state["scale"]
                want[1][b, :, rows] = (ds @ k[:, keys]).view(-1, len(rows), d)
                want[2][b].index_add_(1, keys, ds.transpose(1, 2) @ q.flatten(1, 2))
                want[3][b].index_add_(1, keys, p.transpose(1, 2) @ do)
    return tuple(want) if train else want[0]
