"""Calls on tensors of a device that is not the current one: the library is entered with that device current and a stream of it.  On the CPU, with
tensors that say they are on cuda:1, a current device and streams that only keep count, and a library that records."""
import contextlib

import pytest
import torch

import paper_2505_14687_amd as grat
from paper_2505_14687_amd import grat as grid_binding
from paper_2505_14687_amd import probe
from paper_2505_14687_amd import sequence as sq

THERE = torch.device("cuda", 1)


class There(torch.Tensor):
    device = property(lambda self: THERE)
    is_cuda = property(lambda self: True)


class Stream:
    def __init__(self, index):
        self.device, self.device_index, self.cuda_stream = torch.device("cuda", index), index, 100 + index


@pytest.fixture
def calls(monkeypatch):
    """(entry point, current device, stream) of every call into the library."""
    now, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], torch.device(d).index
        yield
        now[0] = before

    class Recorder:
        def __getattr__(self, name):
            def call(*args):
                if not name.endswith("_work"):
                    seen.append((name, now[0], args[-1]))
                return 0
            return call

    empty = torch.empty
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: Stream(now[0] if d is None else torch.device(d).index))
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: empty(*a, **{**kw, "device": "cpu"}).as_subclass(There))
    sq._library()
    real = grid_binding._lib
    monkeypatch.setattr(grid_binding, "_native", grid_binding._NoNative)
    monkeypatch.setattr(sq, "_native", sq._NoNative)
    monkeypatch.setattr(sq, "_lib", Recorder())
    recorder = Recorder()
    recorder.grat_block_list_shape = real.grat_block_list_shape
    monkeypatch.setattr(grid_binding, "_lib", recorder)
    yield seen
    assert now == [0]


def there(*shape, dtype=torch.bfloat16):
    return torch.zeros(shape, dtype=dtype).as_subclass(There)


def entries(stream):
    Q, K, O = there(1, 4, 64, 64), there(1, 2, 64, 64), there(1, 4, 64, 64)
    count, index = there(1, 2, 2, dtype=torch.int32), there(1, 2, 2, 2, dtype=torch.int32)
    means, scores, lse = there(1, 2, 2, 64, dtype=torch.float32), there(1, 2, 2, 2, dtype=torch.float32), there(1, 4, 64, dtype=torch.float32)
    table, start, s = there(64, 32, 2, dtype=torch.float32), there(1, dtype=torch.int32), dict(stream=stream)
    c, i = there(4, dtype=torch.int32), there(4, 9, dtype=torch.int32)
    lists = dict(n_q=64, n_k=64, q_group=32, block=32)
    return {
        "grat_rotary_table": lambda: grat.grat_rotary_table(8, [8], device=THERE, **s),
        "grat_rotary": lambda: grat.grat_rotary(Q, K, table, **s),
        "grat_rotary_append": lambda: grat.grat_rotary_append(Q, K, K, table, K, K, start, **s),
        "grat_block_means": lambda: grat.grat_block_means(K, 32, **s),
        "grat_block_scores": lambda: grat.grat_block_scores(Q, means, 0.1, 32, 32, 64, **s),
        "grat_select_blocks": lambda: grat.grat_select_blocks(scores, 2, 0, 1, **lists, **s),
        "grat_selected_attention_fwd": lambda: grat.grat_selected_attention_fwd(Q, K, K, 0.1, count, index, 32, 32, return_lse=True, **s),
        "grat_selected_attention_bwd": lambda: grat.grat_selected_attention_bwd(Q, Q, K, K, O, lse, 0.1, count, index, 32, 32, **s),
        "grat_build_block_lists": lambda: grat.grat_build_block_lists((8, 8), (4, 4), "block", (1, 1), device=THERE, **s),
        "grat_validate_block_lists": lambda: grat.grat_validate_block_lists((8, 8), (4, 4), c, i, **s),
        "grat_attention_fwd": lambda: grat.grat_attention_fwd(Q, Q, Q, 0.1, (8, 8), (4, 4), c, i, **s),
        "grat_attention_global_fwd": lambda: grat.grat_attention_global_fwd(Q, Q, Q, 0.1, 0, True, (8, 8), (4, 4), c, i, **s),
        "grat_attention_packed_fwd": lambda: grat.grat_attention_packed_fwd(there(1, 64, 3, 4, 64), 0.1, (8, 8), (4, 4), c, i, **s),
        "grat_dense_attention_fwd": lambda: grat.grat_dense_attention_fwd(Q, Q, Q, 0.1, **s),
        "grat_probe_mfma": lambda: probe.grat_probe_mfma(torch.bfloat16, "ones", 1, 1, sink=there(256, dtype=torch.int64), **s),
    }


@pytest.mark.parametrize("name", entries(None))
def test_the_tensors_device_is_current(calls, name):
    entries(None)[name]()
    assert calls == [(name, 1, 101)]


@pytest.mark.parametrize("name", entries(None))
def test_a_stream_of_the_tensors_device(calls, name):
    stream = Stream(1)
    stream.cuda_stream = 777
    entries(stream)[name]()
    assert calls == [(name, 1, 777)]


@pytest.mark.parametrize("name", entries(None))
def test_a_stream_of_another_device_is_refused(calls, name):
    with pytest.raises(ValueError, match="stream"):
        entries(Stream(0))[name]()
    assert not calls
