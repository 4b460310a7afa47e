"""Attention within a window and over caches: what the library and the binding refuse, before any launch (CPU), and that both ways of marshalling come to
the same (GPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2505_14687_amd as grat
from oracle import window_oracle as orc
from paper_2505_14687_amd import sequence as sq
from paper_2505_14687_amd import window as wn
from test_sequence_abi import DIMS, FAKE, NULL, UNSUPPORTED, ref, rotary, seq, tensor

EIGHT = torch.float8_e4m3fn


def scales(data=FAKE, b=0, h=4096, n=1):
    return sq._Tensor(data, b, h, n)


def test_window_refusals():
    L = wn._library()
    t = tensor()

    def fwd(s, q=t, k=t, v=t, o=t, scale=0.1, window=10, sinks=0, work=FAKE):
        return L.grat_window_attention_fwd(ref(s), ref(q), ref(k), ref(v), ref(o), None, scale, window, sinks, work, None)

    def bwd(s, lse=FAKE, dv=t, window=10, sinks=0, work=FAKE, scale=0.1):
        return L.grat_window_attention_bwd(ref(s), *[ref(t)] * 5, lse, ref(t), ref(t), ref(dv), scale, window, sinks, work, None)
    assert fwd(None) == NULL and fwd(seq(), q=None) == NULL and fwd(seq(), o=tensor(None)) == NULL
    assert bwd(None) == NULL and bwd(seq(), lse=None) == NULL and bwd(seq(), work=None) == NULL and bwd(seq(), dv=None) == NULL
    for call in (fwd, bwd):
        for s in (seq(batch=0), seq(q_heads=0), seq(kv_heads=0), seq(q_heads=5), seq(n_q=0), seq(n_k=0), seq(n_q=-1)):
            assert call(s) == DIMS
        assert call(seq(), window=-1) == DIMS and call(seq(), sinks=-1) == DIMS
        for scale in (0.0, -0.1, float("nan"), float("inf")):
            assert call(seq(), scale=scale) == DIMS
        for s in (seq(dtype=1), seq(dtype=7), seq(d=96), seq(d=256), seq(n_q=1 << 30), seq(n_k=1 << 30), seq(batch=40000), seq(q_heads=65536, kv_heads=1),
                  seq(n_q=1 << 27), seq(n_k=1 << 27)):
            assert call(s) == UNSUPPORTED
        assert call(seq(n_k=1 << 22), sinks=(1 << 20) + 1) == UNSUPPORTED
        assert call(seq(), work=FAKE + 4) == UNSUPPORTED
    assert fwd(seq(), k=tensor(n=64)) == DIMS and fwd(seq(), v=tensor(n=132)) == UNSUPPORTED and fwd(seq(), o=tensor(FAKE + 8)) == UNSUPPORTED
    assert fwd(seq(batch=2)) == DIMS and fwd(seq(batch=2), o=tensor(b=4 * 4096 * 128, h=0)) == DIMS           # outputs that repeat
    assert bwd(seq(), dv=tensor(h=0)) == DIMS
    long = seq(n_q=4, n_k=100000)
    assert L.grat_window_attention_work(ref(long), 0, 0, 0) > 0 and fwd(long, window=0, work=None) == NULL    # keys shared by workgroups
    assert L.grat_window_attention_work(ref(seq(d=96)), 10, 0, 1) == 0 and L.grat_window_attention_work(None, 10, 0, 0) == 0
    assert L.grat_window_attention_work(ref(seq()), 10, 0, 1) >= 8 * 4 * 100


def test_work_of_a_gradient_stays_small():
    """Rows that see first keys are cut into parts; all others are their tile's only part where there are many tiles."""
    L = wn._library()
    s = seq(q_heads=32, kv_heads=8, n_q=16384, n_k=16384)
    rows = 8 * 32 * 16384
    parts = 8 * -(-16384 * 4 // 4352) * 2 * 64 * 128 * 4
    assert rows <= L.grat_window_attention_work(ref(s), 1024, 4, 1) <= rows + parts + 4096
    assert rows <= L.grat_window_attention_work(ref(s), 1024, 0, 1) <= rows + 4096


def test_cache_refusals():
    L = wn._library()
    t, e, s = tensor(), tensor(), scales()

    def append(a, q=t, qo=t, k=t, v=t, kc=e, vc=e, ks=s, vs=s, n=50):
        return L.grat_cache_append(*[ref(x) for x in (a, q, qo, k, v, kc, vc, ks, vs)], n, None)
    ok = dict(start=FAKE)
    assert append(None) == NULL and append(rotary()) == NULL                                            # no start
    for bad in (dict(q=None), dict(qo=None), dict(k=None), dict(v=None), dict(kc=None), dict(vc=tensor(None)), dict(ks=None), dict(vs=scales(None))):
        assert append(rotary(**ok), **bad) == NULL
    assert append(rotary(**ok), n=0) == DIMS and append(rotary(inverse=1, **ok)) == DIMS and append(rotary(batch=0, **ok)) == DIMS
    assert append(rotary(rot=130, **ok)) == DIMS and append(rotary(kv_heads=0, **ok)) == DIMS and append(rotary(axes=2, pairs=(64, 0, 0), **ok)) == DIMS
    assert append(rotary(axes=2, pairs=(32, 32, 0), **ok)) == NULL                                       # several axes without positions
    assert append(rotary(**ok), n=1 << 30) == UNSUPPORTED and append(rotary(dtype=7, **ok)) == UNSUPPORTED
    assert append(rotary(d=192, rot=64, pairs=(32, 0, 0), **ok), *[tensor(n=192)] * 6) == UNSUPPORTED
    assert append(rotary(table=FAKE + 4, **ok)) == UNSUPPORTED
    for bad, st in ((tensor(n=64), DIMS), (tensor(n=136), UNSUPPORTED), (tensor(FAKE + 8), UNSUPPORTED), (tensor(h=-16), DIMS), (tensor(h=0), DIMS)):
        assert append(rotary(**ok), kc=bad) == st and append(rotary(**ok), vc=bad) == st
    for bad, st in ((scales(FAKE + 2), UNSUPPORTED), (scales(n=0), DIMS), (scales(n=1 << 24), UNSUPPORTED), (scales(h=0), DIMS), (scales(h=-1), DIMS),
                    (scales(h=1 << 46), UNSUPPORTED)):
        assert append(rotary(**ok), ks=bad) == st and append(rotary(**ok), vs=bad) == st
    assert append(rotary(batch=2, **ok)) == DIMS                                                         # a cache that repeats
    assert append(rotary(**ok), ks=None, vs=None, kc=tensor(n=132)) == UNSUPPORTED                       # of the tensors' own type

    def read(dtype=0, b=1, h=2, n=50, d=128, c=e, sc=s, o=t):
        return L.grat_cache_read(dtype, b, h, n, d, ref(c), ref(sc), None, ref(o), None)
    assert read(c=None) == NULL and read(sc=None) == NULL and read(o=None) == NULL and read(c=tensor(None)) == NULL
    assert read(b=0) == DIMS and read(h=0) == DIMS and read(n=0) == DIMS and read(o=tensor(h=0)) == DIMS and read(c=tensor(n=64)) == DIMS
    assert read(dtype=7) == UNSUPPORTED and read(d=96) == UNSUPPORTED and read(n=1 << 28) == UNSUPPORTED and read(b=70000) == UNSUPPORTED
    assert read(c=tensor(n=136)) == UNSUPPORTED and read(o=tensor(n=132)) == UNSUPPORTED and read(sc=scales(FAKE + 1)) == UNSUPPORTED

    def attend(s_, q=t, kc=e, vc=e, ks=s, vs=s, o=t, scale=0.1, window=0, sinks=0, parent=None, stride=0, work=FAKE):
        return L.grat_cache_attention_fwd(ref(s_), ref(q), ref(kc), ref(vc), ref(ks), ref(vs), ref(o), None, scale, window, sinks, parent, stride, work, None)
    assert attend(None) == NULL
    for bad in (dict(q=None), dict(kc=None), dict(vc=None), dict(ks=None), dict(vs=None), dict(o=None)):
        assert attend(seq(), **bad) == NULL
    assert attend(seq(n_q=257), parent=FAKE) == UNSUPPORTED and attend(seq(), parent=FAKE, stride=-1) == DIMS
    assert attend(seq(), window=-1) == DIMS and attend(seq(), sinks=-2) == DIMS and attend(seq(), scale=0.0) == DIMS and attend(seq(q_heads=3)) == DIMS
    assert attend(seq(dtype=1)) == UNSUPPORTED and attend(seq(d=96)) == UNSUPPORTED and attend(seq(n_k=1 << 27)) == UNSUPPORTED
    assert attend(seq(), kc=tensor(n=136)) == UNSUPPORTED and attend(seq(), ks=scales(n=0)) == DIMS and attend(seq(), work=FAKE + 8) == UNSUPPORTED
    assert attend(seq(), ks=None, vs=None, vc=tensor(n=132)) == UNSUPPORTED and attend(seq(batch=2)) == DIMS
    long = seq(n_q=1, n_k=100000)
    for eight in (0, 1):
        assert L.grat_cache_attention_work(ref(long), 0, 0, eight) > 0
    assert attend(long, work=None) == NULL
    assert L.grat_cache_attention_work(None, 0, 0, 1) == 0 and L.grat_cache_attention_work(ref(seq(d=80)), 0, 0, 1) == 0


def test_binding_refusals():
    Q, K = torch.zeros(1, 4, 100, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 100, 128, dtype=torch.bfloat16)
    lse, C, S = torch.zeros(1, 4, 100), torch.zeros(1, 2, 100, 128).to(EIGHT), torch.zeros(1, 2, 100)
    table, start = torch.zeros(100, 64, 2), torch.zeros(1, dtype=torch.int32)
    both = dict(K_scale=S, V_scale=S)
    for match, call in [
        ("device memory", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, window=4)),
        ("device memory", lambda: grat.grat_window_attention_bwd(Q, Q, K, K, Q, lse, 0.1)),
        ("window", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, window=0)),
        ("window", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, window=2 ** 32 + 1)),
        ("sinks", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, window=4, sinks=-1)),
        ("sinks", lambda: grat.grat_window_attention_bwd(Q, Q, K, K, Q, lse, 0.1, window=4, sinks=2 ** 32)),
        ("share", lambda: grat.grat_window_attention_fwd(Q[:, :3], K, K, 0.1)),
        ("V must have shape", lambda: grat.grat_window_attention_fwd(Q, K, K[:, :, :50], 0.1)),
        ("dtype and the device", lambda: grat.grat_window_attention_fwd(Q, K.half(), K.half(), 0.1)),
        ("contiguous", lambda: grat.grat_window_attention_fwd(Q.transpose(2, 3), K, K, 0.1)),
        ("k_len", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, k_len=torch.zeros(2, dtype=torch.int32))),
        ("q_pos", lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, q_pos=torch.zeros(1))),
        ("lse", lambda: grat.grat_window_attention_bwd(Q, Q, K, K, Q, lse[:, :2], 0.1)),
        ("dO must have shape", lambda: grat.grat_window_attention_bwd(Q[:, :2], Q, K, K, Q, lse, 0.1)),
        ("device memory", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, **both)),
        ("K_cache must be a tensor of torch.float8", lambda: grat.grat_cache_append(Q, K, K, table, K, K, start, **both)),
        ("dtype", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start)),
        ("both", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, K_scale=S)),
        ("scales must be float32", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, K_scale=S[..., :50], V_scale=S)),
        ("scales must be float32", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, K_scale=S, V_scale=S.double())),
        ("start", lambda: grat.grat_cache_append(Q, K, K, table, C, C, None, **both)),
        ("without a table", lambda: grat.grat_cache_append(Q, K, K, None, C, C, start, **both)),
        ("out is Q's", lambda: grat.grat_cache_append(None, K, K, table, C, C, start, out=Q, **both)),
        ("layout", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, layout="other", **both)),
        ("layout", lambda: grat.grat_cache_append(None, K, K, None, C, C, start, layout="other", **both)),
        ("positions", lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, positions=torch.zeros(1, 99, 1, dtype=torch.int32), **both)),
        ("V must have shape", lambda: grat.grat_cache_append(Q, K, K[:, :1], table, C, C, start, **both)),
        ("V_cache must have shape", lambda: grat.grat_cache_append(Q, K, K, table, C, C[:, :, :50], start, K_scale=S, V_scale=S[..., :50])),
        ("device memory", lambda: grat.grat_cache_read(C, S, torch.bfloat16)),
        ("unsupported dtype", lambda: grat.grat_cache_read(C, S, torch.float64)),
        ("scale", lambda: grat.grat_cache_read(C, None, torch.bfloat16)),
        ("cache must be a tensor of torch.float8", lambda: grat.grat_cache_read(K, S, torch.bfloat16)),
        ("k_len", lambda: grat.grat_cache_read(C, S, torch.bfloat16, k_len=torch.zeros(1))),
        ("device memory", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, **both)),
        ("dtype", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1)),
        ("both", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, V_scale=S)),
        ("parent", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, parent=torch.zeros(3, 100, dtype=torch.int32), **both)),
        ("parent", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, parent=torch.zeros(100), **both)),
        ("parent", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, parent=torch.zeros(99, dtype=torch.int32), **both)),
        ("window", lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, window=-3, **both)),
        ("share", lambda: grat.grat_cache_attention_fwd(Q[:, :3], C, C, 0.1, **both)),
    ]:
        with pytest.raises(ValueError, match=match):
            call()


def calls_on(device):
    """name -> (call(tensors), the tensors whose gradient it would lose)"""
    def floats(*shape):
        return torch.zeros(shape, device=device)
    t = dict(Q=floats(1, 4, 9, 128).bfloat16(), K=floats(1, 2, 9, 128).bfloat16(), V=floats(1, 2, 9, 128).bfloat16(), dO=floats(1, 4, 9, 128).bfloat16(),
             O=floats(1, 4, 9, 128).bfloat16(), lse=floats(1, 4, 9), table=floats(9, 64, 2), scale=floats(1, 2, 9), out=floats(1, 4, 9, 128).bfloat16())
    cache, start = floats(1, 2, 9, 128).to(EIGHT), torch.zeros(1, dtype=torch.int32, device=device)
    return t, {
        "fwd": (lambda x: grat.grat_window_attention_fwd(x["Q"], x["K"], x["V"], 0.1, window=3, out=x["out"]), ("Q", "K", "V", "out")),
        "bwd": (lambda x: grat.grat_window_attention_bwd(x["dO"], x["Q"], x["K"], x["V"], x["O"], x["lse"], 0.1, window=3), ("dO", "Q", "K", "V", "O", "lse")),
        "append": (lambda x: grat.grat_cache_append(x["Q"], x["K"], x["V"], x["table"], cache, cache.clone(), start, K_scale=x["scale"],
                                                    V_scale=x["scale"].detach().clone(), out=x["out"]), ("Q", "K", "V", "table", "scale", "out")),
        "read": (lambda x: grat.grat_cache_read(cache, x["scale"], torch.float32), ("scale",)),
        "attend": (lambda x: grat.grat_cache_attention_fwd(x["Q"], cache, cache, 0.1, K_scale=x["scale"], V_scale=x["scale"], out=x["out"]), ("Q", "scale", "out")),
        "attend16": (lambda x: grat.grat_cache_attention_fwd(x["Q"], x["K"], x["V"], 0.1), ("Q", "K", "V")),
    }


def check_gradients_are_not_lost(device):
    tensors, entries = calls_on(device)
    for call, names in entries.values():
        for name in names:
            if device == "cpu" and name == "out":   # (results are looked at when the device is known to be right)
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


def test_the_native_part_leaves_alone_what_is_not_ordinary():
    wn._library()
    n = wn._native
    Q = torch.zeros(1, 4, 100, 128, dtype=torch.bfloat16)   # host tensors
    assert n.window_fwd(Q, Q, Q, 0.1, 4, 0, True, None, None, False, None, None) is None
    assert n.window_bwd(Q, Q, Q, 0.1, 4, 0, True, None, None, Q, Q, Q, None, None) is None
    assert n.cache_append(Q, Q, Q, Q, Q, Q, None, None, None, None, 0, None, None, None) is None
    assert n.cache_read(Q, Q, 0, None, None, None) is None
    assert n.cache_attention(Q, Q, Q, 0.1, None, None, None, None, None, 0, False, None, None) is None
    with pytest.raises(TypeError):
        n.window_fwd(Q)


def test_the_oracle():
    """Small cases by hand; a tree without branches is a chain; values of 8 bits are torch's."""
    assert orc.window_seen(2, 5, 1, 2, 1)[0].tolist() == [[True, False, True, True, False], [True, False, False, True, True]]
    assert orc.window_seen(2, 5, 1, 2, 0, causal=False)[0].tolist() == [[False, False, True, True, True], [False, False, False, True, True]]
    assert orc.tree_seen([[-1, 0, 0]], 5)[0].tolist() == [[True, True, True, False, False], [True, True, True, True, False], [True, True, True, False, True]]
    for window, sinks in ((None, 0), (3, 0), (3, 2), (1, 7)):
        chain = orc.tree_seen([[-1, 0, 1, 2], [-1, 0, 1, 2]], 9, window, sinks, [9, 2])
        assert np.array_equal(chain, orc.window_seen(4, 9, 2, window, sinks, True, [9, 2]))
    x = np.random.default_rng(1).standard_normal(5000) * np.exp2(np.random.default_rng(2).integers(-12, 7, 5000))
    x = np.clip(x, -448, 448).astype(np.float32)
    assert np.array_equal(orc.e4m3(x), torch.from_numpy(x).to(EIGHT).double().numpy())
    values, s = orc.quantise([[448.0, 1.0], [449.0, -3.0], [0.0, 0.0], [np.inf, 2.0 ** -130]])
    assert s.tolist() == [1.0, 2.0, 1.0, 2.0 ** -126] and values[0].tolist() == [448.0, 1.0] and np.isnan(values[3][0])


# ---- on the GPU --------------------------------------------------------------------------------

@pytest.mark.gpu
def test_both_ways_give_the_same_and_refuse_the_same():
    g = torch.Generator(device="cuda").manual_seed(5)
    B, Hq, Hkv, N, M, d = 2, 4, 2, 20, 300, 128
    Q, dO = (torch.randn((B, Hq, N, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    K, V = (torch.randn((B, Hkv, N, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    lens, start = torch.tensor([223, 20], dtype=torch.int32, device="cuda"), torch.tensor([203, 0], dtype=torch.int32, device="cuda")
    up = torch.arange(N, dtype=torch.int32, device="cuda") // 2 - 1
    table = grat.grat_rotary_table(300, [64])
    wn._library()
    here = torch.cuda.current_stream()   # given: the long way

    def run(stream):
        s = dict(stream=stream)
        out = []
        for eight in (False, True):
            kc, vc = (torch.zeros(B, Hkv, M, d, device="cuda").to(EIGHT if eight else torch.bfloat16) for _ in range(2))
            sc = dict(K_scale=torch.ones(B, Hkv, M, device="cuda"), V_scale=torch.ones(B, Hkv, M, device="cuda")) if eight else {}
            q = grat.grat_cache_append(Q, K, V, table, kc, vc, start, layout="interleaved", **sc, **s)
            assert grat.grat_cache_append(None, K, V, table, kc, vc, start, layout="interleaved", **sc, **s) is None
            O, lse = grat.grat_cache_attention_fwd(q, kc, vc, 0.1, k_len=lens, parent=up, window=100, sinks=2, return_lse=True, **sc, **s)
            out += [q, kc.float(), vc.float(), *sc.values(), O, lse, grat.grat_cache_attention_fwd(q, kc, vc, 0.1, k_len=lens, **sc, **s)]
        out.append(grat.grat_cache_read(kc, sc["K_scale"], torch.float16, k_len=lens, **s))
        O, lse = grat.grat_window_attention_fwd(Q, K, V, 0.1, window=7, sinks=1, return_lse=True, **s)
        grads = grat.grat_window_attention_bwd(dO, Q, K, V, O, lse, 0.1, window=7, sinks=1, **s)
        return (*out, O, lse, *grads, grat.grat_window_attention_fwd(Q, K, V, 0.1, causal=False, k_len=start, q_pos=lens, **s))

    native = wn._native
    assert native.window_fwd(Q, K, V, 0.1, 7, 1, True, None, None, False, None, None) is not None
    assert native.window_fwd(Q, K, V, 0.1, 7, 1, True, None, None, False, None, here) is None
    short, long = run(None), run(here)
    torch.cuda.synchronize()
    for i, (x, y) in enumerate(zip(short, long)):
        assert torch.equal(x, y) and x.stride() == y.stride(), i
    C, S = torch.zeros(B, Hkv, M, d, device="cuda").to(EIGHT), torch.ones(B, Hkv, M, device="cuda")
    out = torch.empty_like(Q)
    assert grat.grat_cache_attention_fwd(Q, C, C, 0.1, K_scale=S, V_scale=S, out=out) is out
    read = torch.empty(C.shape, dtype=torch.float32, device="cuda")
    assert grat.grat_cache_read(C, S, torch.float32, out=read) is read
    for stream in (None, here):
        for call, st in [(lambda: grat.grat_window_attention_fwd(Q.float(), K.float(), V.float(), 0.1, stream=stream), UNSUPPORTED),
                         (lambda: grat.grat_window_attention_fwd(Q, K, V, -0.1, stream=stream), DIMS),
                         (lambda: grat.grat_cache_attention_fwd(Q, C[..., :64], C[..., :64], 0.1, K_scale=S, V_scale=S, stream=stream), None),
                         (lambda: grat.grat_cache_read(C[..., :32], S, torch.float32, stream=stream), UNSUPPORTED)]:
            with pytest.raises(ValueError if st is None else grat.GratError) as e:
                call()
            assert st is None or e.value.status == st
        with pytest.raises(ValueError):
            grat.grat_window_attention_fwd(Q, K, V, 0.1, window=0, stream=stream)


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
def test_autograd_notices_what_is_written(given):
    t, _ = calls_on("cuda")
    Q, K, V = t["Q"], t["K"], t["V"]
    kc, vc = torch.zeros(1, 2, 9, 128, device="cuda").to(EIGHT), torch.zeros(1, 2, 9, 128, device="cuda").to(EIGHT)
    ks, vs = torch.zeros(1, 2, 9, device="cuda"), torch.zeros(1, 2, 9, device="cuda")
    start, s = torch.zeros(1, dtype=torch.int32, device="cuda"), dict(stream=torch.cuda.current_stream() if given else None)
    Qo, Ko, Vo, read = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V), torch.empty(1, 2, 9, 128, device="cuda")
    mine = (Q, K, V, kc, vc, ks, vs, Qo, Ko, Vo, read, t["out"])
    sc = dict(K_scale=ks, V_scale=vs, **s)
    for call, written in [
        (lambda: grat.grat_window_attention_fwd(Q, K, V, 0.1, out=t["out"], **s), (t["out"],)),
        (lambda: grat.grat_window_attention_bwd(t["dO"], Q, K, V, t["O"], t["lse"], 0.1, out=(Qo, Ko, Vo), **s), (Qo, Ko, Vo)),
        (lambda: grat.grat_cache_append(Q, K, V, t["table"], kc, vc, start, out=Qo, **sc), (Qo, kc, vc, ks, vs)),
        (lambda: grat.grat_cache_append(None, K, V, t["table"], Ko, Vo, start, **s), (Ko, Vo)),
        (lambda: grat.grat_cache_read(kc, ks, torch.float32, out=read, **s), (read,)),
        (lambda: grat.grat_cache_attention_fwd(Q, kc, vc, 0.1, out=t["out"], **sc), (t["out"],)),
    ]:
        before = [x._version for x in mine]
        call()
        for x, v in zip(mine, before):
            assert x._version - v == any(x is w for w in written)
        with torch.inference_mode():
            call()


def odd(t):
    """The same tensor, with strides 3, 5 and 7 on its axes of one element."""
    n = t.dim() - 1 if t.dim() == 4 else 3
    return t.as_strided(t.shape, [k if size == 1 else s for size, s, k in zip(t.shape[:n], t.stride()[:n], (3, 5, 7))] + list(t.stride()[n:]))


@pytest.mark.gpu
@pytest.mark.parametrize("given", [False, True])
def test_axes_of_one_element_and_inputs_that_repeat(given):
    s = dict(stream=torch.cuda.current_stream() if given else None)
    g = torch.Generator(device="cuda").manual_seed(7)
    x = torch.randn((1, 1, 1, 128), generator=g, device="cuda").bfloat16()
    table, start = grat.grat_rotary_table(4, [64]), torch.zeros(1, dtype=torch.int32, device="cuda")

    def one(f):
        c, sc = f(torch.zeros(1, 1, 1, 128, device="cuda").to(EIGHT)), f(torch.zeros(1, 1, 1, device="cuda"))
        q = grat.grat_cache_append(f(x), f(x), f(x), table, c, f(c.clone()), start, K_scale=sc, V_scale=f(sc.clone()), **s)
        O, lse = grat.grat_window_attention_fwd(f(x), f(x), f(x), 0.1, return_lse=True, **s)
        return (q, c.float(), sc, O, *grat.grat_window_attention_bwd(f(x), f(x), f(x), f(x), f(O), lse, 0.1, **s),
                grat.grat_cache_attention_fwd(f(x), c, c, 0.1, K_scale=sc, V_scale=sc, **s), grat.grat_cache_read(c, sc, torch.float32, **s))
    for a, b in zip(one(lambda t: t), one(odd)):
        assert torch.equal(a, b)
    # one query for all sequences and heads, one K/V head for several, one cache for all sequences
    B, H, M = 3, 4, 100
    q = torch.randn((1, 1, 2, 128), generator=g, device="cuda").half().expand(B, H, 2, 128)
    k = torch.randn((B, 1, M, 128), generator=g, device="cuda").half().expand(B, H, M, 128)
    c = torch.randn((1, H, M, 128), generator=g, device="cuda").to(EIGHT)
    sc = torch.rand((1, H, 1), generator=g, device="cuda")

    def several(f):
        O, lse = grat.grat_window_attention_fwd(f(q), f(k), f(k), 0.1, window=30, return_lse=True, **s)
        cc, ss = f(c.expand(B, H, M, 128)), f(sc.expand(B, H, M)) if f(sc.expand(B, H, M)).stride(2) else sc.expand(1, H, M).contiguous().expand(B, H, M)
        return (O, *grat.grat_window_attention_bwd(O, f(q), f(k), f(k), O, lse, 0.1, window=30, **s),
                grat.grat_cache_attention_fwd(f(q), cc, cc, 0.1, K_scale=ss, V_scale=ss, **s))
    for a, b in zip(several(lambda t: t), several(lambda t: t.contiguous())):
        assert torch.equal(a, b)


@pytest.mark.parametrize("batch,q_heads,kv_heads,n,window,sinks,causal", [
    (8, 32, 8, 16384, 128, 4096, 1), (1, 32, 8, 32768, 64, 8192, 1), (1, 32, 8, 16384, 128, 1024, 1), (1, 32, 8, 16384, 128, 4096, 1), (1, 8, 1, 16384, 128, 4096, 1),
    (4, 32, 32, 16384, 128, 4, 1), (8, 32, 8, 4096, 128, 1000, 1), (2, 16, 2, 8192, 300, 700, 0), (1, 4, 4, 2047, 64, 2000, 1), (1, 1, 1, 1 << 20, 5, 1 << 19, 1),
])
def test_work_of_many_first_keys_stays_small(batch, q_heads, kv_heads, n, window, sinks, causal):
    """The rows that see a tile of first keys are cut into parts until these fill the chip, no further: at most two rounds of 512 workgroups in parts (and one part more a tile), beside
    what the other tiles take where there are few of them (512 parts, and one more a tile); a part's sums are 2 * 64 * head_dim floats."""
    L = wn._library()
    s = seq(batch=batch, q_heads=q_heads, kv_heads=kv_heads, n_q=n, n_k=n, causal=causal)
    heads, tiles, firsts = batch * kv_heads, -(-n // 64), -(-sinks // 64)
    most = (1024 + heads * firsts if heads * firsts < 1024 else 0) + (512 + heads * tiles if heads * tiles < 512 else 0)
    rows = 8 * batch * q_heads * n
    assert rows <= L.grat_window_attention_work(ref(s), window, sinks, 1) <= rows + most * 2 * 64 * 128 * 4 + 4096


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("d,dtype", [(128, 0), (64, 2)])
@pytest.mark.parametrize("shape", [
    dict(batch=1, q_heads=32, kv_heads=32, n_q=1 << 20, n_k=1 << 20), dict(batch=32, q_heads=32, kv_heads=4, n_q=1 << 18, n_k=1 << 20),
    dict(batch=1, q_heads=1, kv_heads=1, n_q=(1 << 28) - 1, n_k=(1 << 28) - 1), dict(batch=1, q_heads=1, kv_heads=1, n_q=(1 << 29) - 1, n_k=5),
    dict(batch=1, q_heads=1, kv_heads=1, n_q=1, n_k=(1 << 28) - 1), dict(batch=255, q_heads=257, kv_heads=257, n_q=4000, n_k=4000),
    dict(batch=1, q_heads=65535, kv_heads=65535, n_q=8191, n_k=4095), dict(batch=1, q_heads=65535, kv_heads=1, n_q=8192, n_k=1 << 20),
    dict(batch=1, q_heads=65, kv_heads=1, n_q=(1 << 29) // 65 - 1, n_k=1 << 20), dict(batch=1, q_heads=129, kv_heads=1, n_q=(1 << 29) // 129 - 1, n_k=1 << 20),
    dict(batch=127, q_heads=129 * 4, kv_heads=4, n_q=(1 << 29) // (127 * 129 * 4), n_k=200000),
])
def test_the_gradient_takes_what_the_forward_call_takes(shape, d, dtype, eight):
    """Up to the limits that the header names no size is refused.  (A tensor is missing: only what is looked at ahead of it can refuse the call.)"""
    L = wn._library()
    t, e, sc = tensor(n=d), tensor(n=d), scales()
    s = seq(d=d, dtype=dtype, **shape)
    for causal in (1, 0):
        s.causal = causal
        for window, sinks in ((0, 0), (1, 0), (128, 4), (2 ** 31 - 1, 1), (64, min(shape["n_k"] - 1, 1 << 19)), (4096, min(shape["n_k"] - 1, 1 << 20)), (300, 2 ** 31 - 1)):
            assert L.grat_window_attention_fwd(ref(s), None, ref(t), ref(t), ref(t), None, 0.1, window, sinks, FAKE, None) == NULL
            assert L.grat_window_attention_bwd(ref(s), None, *[ref(t)] * 4, FAKE, *[ref(t)] * 3, 0.1, window, sinks, FAKE, None) == NULL
            assert L.grat_window_attention_work(ref(s), window, sinks, 1) >= 8 * shape["batch"] * shape["q_heads"] * shape["n_q"]
            kv = (ref(e), ref(e), ref(sc), ref(sc)) if eight else (ref(t), ref(t), None, None)
            assert L.grat_cache_attention_fwd(ref(s), None, *kv, ref(t), None, 0.1, window, sinks, None, 0, FAKE, None) == NULL


def test_tiles_of_prompts_follow_what_was_measured():
    """Scratch memory tells the tiles: 2 048 tokens of 8 heads make 128 of 128 rows, two parts each, or 256 of 64 rows in one part."""
    L = wn._library()
    for d, windows in ((128, {1500: 64, 1800: 64, 2100: 128}), (64, {2500: 64, 3200: 128})):
        s = seq(d=d, q_heads=8, kv_heads=8, n_q=2048, n_k=8192)
        for window, tile in windows.items():
            assert L.grat_window_attention_work(ref(s), window, 0, 0) == (0 if tile == 64 else 2 * 128 * 128 * (d + 2) * 4), (d, window)


@pytest.mark.parametrize("eight", [0, 1])
@pytest.mark.parametrize("batch,heads,n_q,window,sinks,d", [
    (4, 8, 64, 256, 16384, 128), (1, 8, 64, 256, 16384, 128), (4, 8, 64, 256, 1025, 128), (4, 8, 64, 64, 1985, 128), (8, 8, 40, 100, 6005, 128), (4, 8, 64, 63, 2050, 64),
    (1, 2, 600, 129, 8001, 128), (1, 2, 700, 129, 8001, 64),
])
def test_tiles_count_first_keys(batch, heads, n_q, window, sinks, d, eight):
    """Rows that see many first keys and a short window are worked on as rows that see as many keys near them.  (Scratch memory tells the tiles.)"""
    L = wn._library()
    both = batch, 4 * heads, heads
    mine = seq(0, *both, d=d, n_q=n_q, n_k=1 << 15)
    same = seq(0, *both, d=d, n_q=n_q, n_k=window - 1 + n_q + sinks)
    assert L.grat_cache_attention_work(ref(mine), window, sinks, eight) == L.grat_cache_attention_work(ref(same), 0, 0, eight) > 0
