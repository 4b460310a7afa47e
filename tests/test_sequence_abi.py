"""Token sequences: what the library and the binding refuse, before any launch (CPU), and that both ways of marshalling come to the
same (GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from paper_2505_14687_amd import sequence as sq

FAKE = 0x1000   # never dereferenced: every call below fails validation first
NULL, DIMS, PATTERN, SMALL, UNSUPPORTED = 1, 2, 4, 5, 6


def tensor(data=FAKE, b=0, h=4096 * 128, n=128):
    return sq._Tensor(data, b, h, n)


def seq(dtype=0, batch=1, q_heads=4, kv_heads=2, d=128, n_q=100, n_k=100, q_group=32, block=64, causal=1):
    return sq._Sequence(dtype, batch, q_heads, kv_heads, d, n_q, n_k, q_group, block, causal, None, None)


def rotary(dtype=0, batch=1, q_heads=4, kv_heads=2, d=128, n=10, rot=128, axes=1, pairs=(64, 0, 0), table=FAKE, n_pos=10, positions=None,
           stride=0, start=None, inverse=0):
    return sq._Rotary(dtype, batch, q_heads, kv_heads, d, n, rot, 0, inverse, axes, (ctypes.c_int32 * 3)(*pairs), table, n_pos, positions, stride, start)


def ref(x):
    return None if x is None else ctypes.byref(x)


def test_rotary_refusals():
    L = sq._library()
    t = tensor()

    def call(a, q=t, qo=t, k=t, ko=t):
        return L.grat_rotary(ref(a), ref(q), ref(qo), ref(k), ref(ko), None)
    assert call(None) == NULL and call(rotary(), q=None) == NULL and call(rotary(), ko=None) == NULL and call(rotary(table=None)) == NULL
    assert call(rotary(), qo=tensor(None)) == NULL
    assert call(rotary(batch=0)) == DIMS and call(rotary(n=0)) == DIMS and call(rotary(rot=130)) == DIMS and call(rotary(n_pos=0)) == DIMS
    assert call(rotary(pairs=(63, 0, 0))) == DIMS and call(rotary(axes=4)) == DIMS and call(rotary(axes=2, pairs=(64, 0, 0))) == DIMS
    assert call(rotary(axes=2, pairs=(32, 32, 0))) == NULL                       # several axes without positions
    assert call(rotary(kv_heads=0)) == DIMS and call(rotary(stride=-1, positions=FAKE)) == DIMS
    assert call(rotary(rot=8, pairs=(4, 0, 0))) == UNSUPPORTED and call(rotary(dtype=5)) == UNSUPPORTED
    assert call(rotary(d=1040, rot=128), q=tensor(n=1040)) == UNSUPPORTED and call(rotary(table=FAKE + 4)) == UNSUPPORTED
    assert call(rotary(), q=tensor(n=64)) == DIMS and call(rotary(), q=tensor(n=132)) == UNSUPPORTED and call(rotary(), k=tensor(FAKE + 2)) == UNSUPPORTED

    def append(a, n_cache=5, v=t):
        return L.grat_rotary_append(ref(a), ref(t), ref(t), ref(t), ref(v), ref(t), ref(t), n_cache, None)
    assert append(rotary()) == NULL and append(rotary(start=FAKE), v=None) == NULL           # no start; no V
    assert append(rotary(start=FAKE), n_cache=0) == DIMS and append(rotary(start=FAKE, inverse=1)) == DIMS
    assert append(rotary(start=FAKE, positions=FAKE)) == DIMS

    def table(scaling=0, base=1e4, factor=1.0, magnitude=1.0, trained=0.0, low=1.0, high=32.0, n_pos=4, axes=1, pairs=(8, 8, 8), out=FAKE):
        spec = sq._Spec(scaling, base, factor, magnitude, trained, low, high)
        return L.grat_rotary_table(ctypes.byref(spec), n_pos, axes, (ctypes.c_int32 * 3)(*pairs), out, None)
    assert table(out=None) == NULL and table(n_pos=0) == DIMS and table(axes=0) == DIMS and table(pairs=(0, 8, 8)) == DIMS
    assert table(scaling=7) == PATTERN and table(base=0.0) == DIMS and table(magnitude=float("inf")) == DIMS
    assert table(scaling=1, factor=0.0) == DIMS and table(scaling=3, trained=0.0) == DIMS
    assert table(scaling=3, trained=10.0, low=2.0, high=2.0) == DIMS
    assert table(pairs=(600, 1, 1)) == UNSUPPORTED and table(n_pos=1 << 28, pairs=(64, 1, 1)) == UNSUPPORTED


def test_list_refusals():
    L = sq._library()
    t = tensor()

    def means(s=seq(), k=t, new=0, out=FAKE):
        return L.grat_block_means(ref(s), ref(k), new, out, None)
    assert means(s=None) == NULL and means(k=None) == NULL and means(out=None) == NULL and means(new=-1) == DIMS
    assert means(s=seq(block=0)) == DIMS and means(s=seq(block=48)) == UNSUPPORTED and means(s=seq(block=8192)) == UNSUPPORTED
    assert means(s=seq(d=96)) == UNSUPPORTED and means(s=seq(dtype=3)) == UNSUPPORTED and means(s=seq(batch=65536)) == UNSUPPORTED
    assert means(s=seq(n_k=1 << 30)) == UNSUPPORTED and means(k=tensor(n=1 << 24)) == UNSUPPORTED

    def scores(s=seq(), q=t, m=FAKE, scale=1.0, out=FAKE, work=FAKE):
        return L.grat_block_scores(ref(s), ref(q), m, scale, out, work, None)
    assert scores(s=None) == NULL and scores(m=None) == NULL and scores(out=None) == NULL and scores(work=None) == NULL
    assert scores(scale=float("nan")) == DIMS and scores(s=seq(kv_heads=3)) == DIMS and scores(s=seq(q_group=0)) == DIMS
    assert scores(s=seq(d=32)) == UNSUPPORTED and scores(work=FAKE + 8) == UNSUPPORTED
    assert L.grat_block_scores_work(ref(seq(n_q=8))) == 0 and L.grat_block_scores_work(ref(seq(n_q=100))) == 2 * 4 * 128 * 4
    assert L.grat_block_scores_work(None) == 0

    def select(s=seq(), x=FAKE, top=4, first=1, local=2, c=FAKE, i=FAKE):
        return L.grat_select_blocks(ref(s), x, top, first, local, c, i, None)
    assert select(s=None) == NULL and select(x=None) == NULL and select(c=None) == NULL and select(i=None) == NULL
    assert select(top=0) == DIMS and select(first=-1) == DIMS and select(first=3) == DIMS and select(local=2 ** 31 - 1) == DIMS
    assert select(top=9000) == UNSUPPORTED and select(s=seq(n_k=32 * 32768 + 1, block=32)) == UNSUPPORTED
    assert select(s=seq(batch=1 << 10, n_q=1 << 16, q_group=1)) == UNSUPPORTED


def test_attention_refusals():
    L = sq._library()
    t = tensor()

    def fwd(s=seq(), q=t, k=t, v=t, o=t, scale=0.1, c=FAKE, i=FAKE, top=4, work=FAKE):
        return L.grat_selected_attention_fwd(ref(s), ref(q), ref(k), ref(v), ref(o), None, scale, c, i, top, work, None)

    def bwd(s=seq(), do=t, dq=t, dk=t, lse=FAKE, scale=0.1, c=FAKE, i=FAKE, top=4, work=FAKE):
        return L.grat_selected_attention_bwd(ref(s), ref(do), ref(t), ref(t), ref(t), ref(t), lse, ref(dq), ref(dk), ref(t), scale, c, i, top, work, None)
    assert fwd(s=None) == NULL and fwd(q=None) == NULL and fwd(o=tensor(None)) == NULL and fwd(c=None) == NULL and fwd(i=None) == NULL
    assert bwd(s=None) == NULL and bwd(do=None) == NULL and bwd(lse=None) == NULL and bwd(dk=None) == NULL and bwd(work=None) == NULL
    for call in (fwd, bwd):
        assert call(scale=0.0) == DIMS and call(scale=float("inf")) == DIMS and call(s=seq(n_q=0)) == DIMS and call(s=seq(q_heads=3)) == DIMS
        assert call(top=0) == SMALL
        assert call(s=seq(dtype=1)) == UNSUPPORTED and call(s=seq(d=96)) == UNSUPPORTED and call(s=seq(block=16)) == UNSUPPORTED
        assert call(top=(1 << 18) // 64 + 1) == UNSUPPORTED and call(work=FAKE + 4) == UNSUPPORTED
        assert call(s=seq(q_heads=65534, n_q=1 << 16, q_group=1 << 16)) == UNSUPPORTED
    assert fwd(k=tensor(n=132)) == UNSUPPORTED and fwd(v=tensor(n=1 << 24)) == UNSUPPORTED and fwd(q=tensor(b=-8)) == DIMS
    # few workgroups share lists that are long, and need room for the parts; many workgroups and short lists do not
    assert fwd(s=seq(n_k=4096), top=32, work=None) == NULL
    assert L.grat_selected_attention_work(ref(seq(batch=64, n_q=512, n_k=4096)), 32, 0) == 0
    assert L.grat_selected_attention_work(ref(seq()), 4, 0) == 0 and L.grat_selected_attention_work(ref(seq(n_k=4096)), 4, 0) == 0
    assert L.grat_selected_attention_work(ref(seq(n_k=4096)), 32, 0) > 0 and L.grat_selected_attention_work(ref(seq()), 4, 1) > 0
    assert L.grat_selected_attention_work(ref(seq(d=96)), 4, 1) == 0 and L.grat_selected_attention_work(None, 4, 0) == 0


@pytest.mark.parametrize("block,top", [(32, 32), (64, 16), (128, 8), (256, 8), (1024, 4), (4096, 2), (4096, 4)])
@pytest.mark.parametrize("n_q,n_k", [(16384, 16384), (1024, 8192), (131072, 131072)])
def test_scratch_of_the_gradient_goes_with_its_results(block, top, n_q, n_k):
    """Parts of the walk over keys hold whole blocks in fp32: twice dK and dV, and as much again for the parts' uneven ends; or, in small launches, 2 * 768 + 1
    parts of 64 keys.  The rest: statistics, lists and bits."""
    s = seq(q_heads=32, kv_heads=8, n_q=n_q, n_k=n_k, q_group=64, block=block)
    results = 2 * 2 * 8 * n_k * 128
    work = sq._library().grat_selected_attention_work(ref(s), top, 1)
    assert work <= 4.25 * results + (2 * 768 + 1) * 64 * 2 * 128 * 4


def test_binding_refusals():
    Q, K = torch.zeros(1, 4, 100, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 100, 128, dtype=torch.bfloat16)
    count, index = torch.zeros(1, 2, 4, dtype=torch.int32), torch.zeros(1, 2, 4, 3, dtype=torch.int32)
    table = torch.zeros(100, 64, 2)

    def attend(q=Q, k=K, v=K, c=count, i=index, **kw):
        return grat.grat_selected_attention_fwd(q, k, v, 0.1, c, i, 32, 64, **kw)
    for bad, match in [(dict(q=Q[0]), "B, H, N, d"), (dict(v=K[:, :, :50]), "shape"), (dict(k=K.half()), "dtype"), (dict(q=Q.double()), "dtype"),
                       (dict(c=count.long()), "int32"), (dict(c=count[:, :, :3]), "shape"), (dict(i=index[:, :1]), "shape"),
                       (dict(i=index.transpose(2, 3)), "shape"), (dict(k=K.repeat(1, 2, 1, 1)[:, :3], v=K.repeat(1, 2, 1, 1)[:, :3]), "share"),
                       (dict(k_len=torch.zeros(2, dtype=torch.int32)), "k_len"), (dict(q_pos=torch.zeros(1)), "q_pos"), ({}, "device memory")]:
        with pytest.raises(ValueError, match=match):
            attend(**bad)
    lse = torch.zeros(1, 4, 100)
    with pytest.raises(ValueError, match="lse"):
        grat.grat_selected_attention_bwd(Q, Q, K, K, Q, lse[:, :2], 0.1, count, index, 32, 64)
    with pytest.raises(ValueError, match="dO"):
        grat.grat_selected_attention_bwd(Q[:, :2], Q, K, K, Q, lse, 0.1, count, index, 32, 64)
    for bad, match in [(dict(layout="thirds"), "layout"), (dict(table=table.half()), "table"), (dict(table=torch.zeros(100, 65, 2)), "pairs"),
                       (dict(axis_pairs=[30, 30]), "axis_pairs"), (dict(axis_pairs=[32, 32]), "positions"),
                       (dict(positions=torch.zeros(1, 99, 1, dtype=torch.int32)), "positions"),
                       (dict(positions=torch.zeros(1, 100, 1, dtype=torch.int32), start=torch.zeros(1, dtype=torch.int32)), "exclude"),
                       ({}, "device memory")]:
        with pytest.raises(ValueError, match=match):
            grat.grat_rotary(Q, K, **{"table": table, **bad})
    with pytest.raises(ValueError, match="scaling"):
        grat.grat_rotary_table(4, [8], scaling="yes")
    with pytest.raises(ValueError, match="axis_pairs"):
        grat.grat_rotary_table(4, [])
    with pytest.raises(ValueError, match="out"):
        grat.grat_block_means(K, 64, new=1)
    with pytest.raises(ValueError, match="means"):
        grat.grat_block_scores(Q, torch.zeros(1, 2, 3, 128), 0.1, 32, 64, 100)
    with pytest.raises(ValueError, match="scores"):
        grat.grat_select_blocks(torch.zeros(1, 2, 4, 3), 2, 0, 1, n_q=100, n_k=100, q_group=32, block=64)
    with pytest.raises(ValueError, match="start"):
        grat.grat_rotary_append(Q, K, K, table, K, K, None)


def test_outputs_whose_rows_lie_on_each_other_are_refused():
    L = sq._library()
    t = tensor(b=4 * 4096 * 128)
    for flat in (tensor(b=0), tensor(b=4 * 4096 * 128, h=0)):
        a, s = rotary(batch=2, start=FAKE), seq(batch=2)
        assert L.grat_rotary(ref(a), ref(t), ref(flat), ref(t), ref(t), None) == DIMS
        assert L.grat_rotary(ref(a), ref(t), ref(t), ref(t), ref(flat), None) == DIMS
        for k in (1, 4, 5):   # Q_out, K_cache, V_cache
            x = [ref(flat if i == k else t) for i in range(6)]
            assert L.grat_rotary_append(ref(a), *x, 5, None) == DIMS
        assert L.grat_selected_attention_fwd(ref(s), ref(t), ref(t), ref(t), ref(flat), None, 0.1, FAKE, FAKE, 4, FAKE, None) == DIMS
        for k in range(3):
            grads = [ref(flat if i == k else t) for i in range(3)]
            assert L.grat_selected_attention_bwd(ref(s), *[ref(t)] * 5, FAKE, *grads, 0.1, FAKE, FAKE, 4, FAKE, None) == DIMS


def test_launches_of_2_to_the_32_threads_are_refused():
    """An axis of a launch ends there: the call says so ahead of it."""
    L = sq._library()
    t = tensor()

    def select(n_k, lists, block=32):
        s = seq(batch=1 << 10, kv_heads=1, q_heads=1, n_q=lists >> 10, n_k=n_k, q_group=1, block=block)
        return L.grat_select_blocks(ref(s), FAKE, 4, 1, 2, FAKE, FAKE, None)
    assert select(32 * 2049, 1 << 24) == UNSUPPORTED and select(32 * 16384, 1 << 24) == UNSUPPORTED      # four waves a list
    assert select(32 * 16385, 1 << 23) == UNSUPPORTED and select(32 * 32768, 1 << 23) == UNSUPPORTED     # eight
    s = seq(batch=1, kv_heads=1, q_heads=1, n_q=(1 << 26) - 3, n_k=64, q_group=1, block=32)              # one, four lists a workgroup
    assert L.grat_select_blocks(ref(s), FAKE, 1, 0, 1, FAKE, FAKE, None) == UNSUPPORTED
    assert L.grat_block_means(ref(seq(n_k=1 << 29, block=32)), ref(t), 0, FAKE, None) == UNSUPPORTED
    for dtype, d, tokens in ((0, 128, 1 << 29), (1, 128, 1 << 28), (0, 1024, 1 << 26), (1, 96, 21 << 24)):
        a = rotary(dtype=dtype, d=d, rot=16, pairs=(8, 0, 0), n=tokens)
        q = tensor(n=d)
        assert L.grat_rotary(ref(a), ref(q), ref(q), None, None, None) == UNSUPPORTED


def test_sizes_that_do_not_fit_32_bits_are_refused():
    """Cut off on the way, 2^32 + 64 keys a block would be 64 with results allocated for one block."""
    Q, K = torch.zeros(1, 4, 100, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 100, 128, dtype=torch.bfloat16)
    much = 2 ** 32 + 64
    count, index = torch.zeros(1, 2, 1, dtype=torch.int32), torch.zeros(1, 2, 1, 3, dtype=torch.int32)
    scores, lse = torch.zeros(1, 2, 4, 2), torch.zeros(1, 4, 100)
    lists = dict(n_q=100, n_k=100, q_group=32, block=64)
    for name, call in [
        ("block", lambda: grat.grat_block_means(K, much)),
        ("new", lambda: grat.grat_block_means(K, 64, new=2 ** 32, out=torch.zeros(1, 2, 2, 128))),
        ("q_group", lambda: grat.grat_block_scores(Q, torch.zeros(1, 2, 2, 128), 0.1, much, 64, 100)),
        ("n_k", lambda: grat.grat_block_scores(Q, torch.zeros(1, 2, 2, 128), 0.1, 32, 64, 2 ** 32 + 100)),
        ("q_group", lambda: grat.grat_select_blocks(scores, 2, 0, 1, **{**lists, "q_group": much})),
        ("block", lambda: grat.grat_select_blocks(scores, 2, 0, 1, **{**lists, "block": much})),
        ("top", lambda: grat.grat_select_blocks(scores, much, 0, 1, **lists)),
        ("first", lambda: grat.grat_select_blocks(scores, 2, 2 ** 32, 1, **lists)),
        ("local", lambda: grat.grat_select_blocks(scores, 2, 0, -2 ** 32, **lists)),
        ("q_group", lambda: grat.grat_selected_attention_fwd(Q, K, K, 0.1, count, index, much, 64)),
        ("block", lambda: grat.grat_selected_attention_fwd(Q, K, K, 0.1, count, index, 100, much)),
        ("q_group", lambda: grat.grat_selected_attention_bwd(Q, Q, K, K, Q, lse, 0.1, count, index, much, 64)),
        ("n_pos", lambda: grat.grat_rotary_table(2 ** 32 + 1, [8])),
        ("Q", lambda: grat.grat_rotary(Q.expand(2 ** 32 + 1, -1, -1, -1), None, torch.zeros(100, 64, 2))),
    ]:
        with pytest.raises(ValueError, match=rf"^{name}\b"):
            call()


def calls_on(device, dtype=torch.bfloat16):
    """name -> (call(tensors), the tensors whose gradient it would lose)"""
    def floats(*shape):
        return torch.zeros(shape, device=device)
    t = dict(Q=floats(1, 4, 100, 128).to(dtype), K=floats(1, 2, 100, 128).to(dtype), V=floats(1, 2, 100, 128).to(dtype),
             dO=floats(1, 4, 100, 128).to(dtype), O=floats(1, 4, 100, 128).to(dtype), table=floats(100, 64, 2), means=floats(1, 2, 2, 128),
             lse=floats(1, 4, 100), cache=floats(1, 2, 100, 128).to(dtype), out=floats(1, 4, 100, 128).to(dtype), kept=floats(1, 2, 2, 128),
             written=floats(1, 2, 4, 2))
    lists = torch.zeros(1, 2, 4, dtype=torch.int32, device=device), torch.full((1, 2, 4, 2), -1, dtype=torch.int32, device=device)
    start = torch.zeros(1, dtype=torch.int32, device=device)
    return t, {
        "rotary": (lambda x: grat.grat_rotary(x["Q"], x["K"], x["table"], out=(x["out"], torch.empty_like(x["K"]))), ("Q", "K", "table", "out")),
        "append": (lambda x: grat.grat_rotary_append(x["Q"], x["K"], x["V"], x["table"], x["cache"], torch.empty_like(x["cache"]), start),
                   ("Q", "K", "V", "table", "cache")),
        "means": (lambda x: grat.grat_block_means(x["K"], 64, out=x["kept"]), ("K", "kept")),
        "scores": (lambda x: grat.grat_block_scores(x["Q"], x["means"], 0.1, 32, 64, 100, out=x["written"]), ("Q", "means", "written")),
        "fwd": (lambda x: grat.grat_selected_attention_fwd(x["Q"], x["K"], x["V"], 0.1, *lists, 32, 64, out=x["out"]), ("Q", "K", "V", "out")),
        "bwd": (lambda x: grat.grat_selected_attention_bwd(x["dO"], x["Q"], x["K"], x["V"], x["O"], x["lse"], 0.1, *lists, 32, 64),
                ("dO", "Q", "K", "V", "O", "lse")),
    }


def check_gradients_are_not_lost(device):
    tensors, entries = calls_on(device)
    for call, names in entries.values():
        for name in names:
            if device == "cpu" and name in ("out", "kept", "written"):   # (results are looked at when the device is known to be right)
                continue
            x = {k: v.clone().requires_grad_(k == name) for k, v in tensors.items()}
            with pytest.raises(ValueError, match="requires a gradient"):
                call(x)
            if device == "cuda":
                with torch.no_grad():
                    call(x)
            with torch.autograd.forward_ad.dual_level():
                x = {k: torch.autograd.forward_ad.make_dual(v, torch.ones_like(v)) if k == name else v for k, v in tensors.items()}
                with pytest.raises(ValueError, match="requires a gradient"):
                    call(x)
        if device == "cuda":
            call(tensors)


def test_gradients_are_not_lost():
    check_gradients_are_not_lost("cpu")


@pytest.mark.gpu
def test_gradients_are_not_lost_on_the_gpu():
    check_gradients_are_not_lost("cuda")
    scores = torch.zeros(1, 2, 4, 2, device="cuda", requires_grad=True)   # lists have no gradient to lose
    count, _ = grat.grat_select_blocks(scores, 1, 0, 0, n_q=100, n_k=100, q_group=32, block=64)
    assert (count == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
def test_autograd_notices_what_is_written(given):
    """Tensors of the caller's that a call writes to have a new version afterwards; in both ways of marshalling."""
    t, _ = calls_on("cuda")
    Q, K, V = t["Q"], t["K"], t["V"]
    lists = torch.zeros(1, 2, 4, dtype=torch.int32, device="cuda"), torch.full((1, 2, 4, 2), -1, dtype=torch.int32, device="cuda")
    start, s = torch.zeros(1, dtype=torch.int32, device="cuda"), dict(stream=torch.cuda.current_stream() if given else None)
    Qo, Ko, Vo = (torch.empty_like(x) for x in (Q, K, V))
    for call, written in [
        (lambda: grat.grat_rotary(Q, K, t["table"], out=(Qo, Ko), **s), (Qo, Ko)),
        (lambda: grat.grat_rotary(Q, None, t["table"], out=(Qo, None), **s), (Qo,)),
        (lambda: grat.grat_rotary_append(Q, K, V, t["table"], t["cache"], Vo, start, out=Qo, **s), (t["cache"], Vo, Qo)),
        (lambda: grat.grat_block_means(K, 64, out=t["kept"], **s), (t["kept"],)),
        (lambda: grat.grat_block_scores(Q, t["means"], 0.1, 32, 64, 100, out=t["written"], **s), (t["written"],)),
        (lambda: grat.grat_selected_attention_fwd(Q, K, V, 0.1, *lists, 32, 64, out=t["out"], **s), (t["out"],)),
        (lambda: grat.grat_selected_attention_fwd(Q, K, V, 0.1, *lists, 32, 64, out=t["out"], return_lse=True, **s), (t["out"],)),
        (lambda: grat.grat_selected_attention_bwd(t["dO"], Q, K, V, t["O"], t["lse"], 0.1, *lists, 32, 64, out=(Qo, Ko, Vo), **s), (Qo, Ko, Vo)),
    ]:
        before = {id(x): x._version for x in (*t.values(), Qo, Ko, Vo)}
        call()
        for x in (*t.values(), Qo, Ko, Vo):
            assert x._version - before[id(x)] == any(x is w for w in written)
        with torch.inference_mode():
            call()
    w = torch.ones(1, 4, 100, 128, dtype=torch.bfloat16, device="cuda", requires_grad=True)
    y = (w * Qo).sum()                       # (saves Qo)
    grat.grat_rotary(Q, None, t["table"], out=(Qo, None), **s)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    with torch.inference_mode():             # these have no version
        a, b = torch.zeros_like(Q), torch.zeros_like(Q)
    grat.grat_rotary(a, None, t["table"], out=(b, None), **s)


def test_the_native_part_leaves_alone_what_is_not_ordinary():
    sq._library()
    n = sq._native
    Q = torch.zeros(1, 4, 100, 128, dtype=torch.bfloat16)   # host tensors
    i = torch.zeros(1, 4, 100, 1, dtype=torch.int32)
    assert n.rotary(Q, None, Q, None, None, 0, None, False, None, None) is None
    assert n.append(Q, Q, Q, Q, Q, Q, None, 0, None, None) is None
    assert n.means(Q, 64, None, 0, None, None) is None
    assert n.scores(Q, Q, 0.1, 1, 64, 100, True, None, None, None, None) is None
    assert n.select(Q, 1, 0, 0, 100, 100, 1, 64, True, None, None, None) is None
    assert n.selected_fwd(Q, Q, Q, 0.1, i, i, 1, 64, True, None, None, False, None, None) is None
    assert n.selected_bwd(Q, Q, Q, 0.1, i, i, 1, 64, True, None, None, Q, Q, Q, None, None) is None
    with pytest.raises(TypeError):
        n.means(Q)


@pytest.mark.gpu
def test_both_ways_give_the_same_and_refuse_the_same():
    g = torch.Generator(device="cuda").manual_seed(5)
    B, Hq, Hkv, N, d = 2, 4, 2, 200, 128
    Q, dO = (torch.randn((B, Hq, N, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    K, V = (torch.randn((B, Hkv, N, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    lens, start = torch.tensor([200, 77], dtype=torch.int32, device="cuda"), torch.tensor([3, 0], dtype=torch.int32, device="cuda")
    table = grat.grat_rotary_table(300, [64])
    sq._library()
    here = torch.cuda.current_stream()   # given: the long way

    def run(stream):
        q, k = grat.grat_rotary(Q, K, table, start=start, stream=stream)
        kc, vc = torch.zeros(B, Hkv, 300, d, device="cuda").bfloat16(), torch.zeros(B, Hkv, 300, d, device="cuda").bfloat16()
        q2 = grat.grat_rotary_append(Q, K, V, table, kc, vc, start, layout="interleaved", stream=stream)
        means = grat.grat_block_means(k, 32, k_len=lens, stream=stream)
        scores = grat.grat_block_scores(q, means, 0.1, 16, 32, N, k_len=lens, stream=stream)
        lists = grat.grat_select_blocks(scores, 4, 1, 2, n_q=N, n_k=N, q_group=16, block=32, k_len=lens, stream=stream)
        O, lse = grat.grat_selected_attention_fwd(q, k, V, 0.1, *lists, 16, 32, k_len=lens, return_lse=True, stream=stream)
        grads = grat.grat_selected_attention_bwd(dO, q, k, V, O, lse, 0.1, *lists, 16, 32, k_len=lens, stream=stream)
        return (q, k, q2, kc, vc, means, scores, *lists, O, lse, *grads)

    native = sq._native
    assert native.means(K, 32, lens, 0, None, None) is not None and native.means(K, 32, lens, 0, None, here) is None
    short, long = run(None), run(here)
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(short, long)):
        assert torch.equal(x, y) and x.stride() == y.stride(), i
    # given outputs come back as they are
    out = torch.empty_like(Q), torch.empty_like(K)
    got = grat.grat_rotary(Q, K, table, start=start, out=out)
    assert got[0] is out[0] and got[1] is out[1] and torch.equal(out[0], short[0])
    alone = grat.grat_rotary(Q, None, table, start=start)
    assert alone[1] is None and torch.equal(alone[0], short[0])
    # the library's refusals arrive as errors either way
    for stream in (None, here):
        with pytest.raises(grat.GratError) as e:
            grat.grat_block_means(K, 48, stream=stream)
        assert e.value.status == UNSUPPORTED
        with pytest.raises(grat.GratError) as e:
            grat.grat_select_blocks(short[6], 2, 2, 2, n_q=N, n_k=N, q_group=16, block=32, stream=stream)
        assert e.value.status == DIMS
        with pytest.raises(grat.GratError) as e:
            grat.grat_selected_attention_fwd(Q.float(), K.float(), V.float(), 0.1, short[7], short[8], 16, 32, stream=stream)
        assert e.value.status == UNSUPPORTED
        with pytest.raises(ValueError):
            grat.grat_selected_attention_fwd(Q, K, V, 0.1, short[7], short[8].long(), 16, 32, stream=stream)
