"""Calls on tensors of a device that is not the current one (see test_devices.py): attention within a window and over caches."""
import pytest
import torch

import paper_2505_14687_amd as grat
from paper_2505_14687_amd import sequence as sq
from paper_2505_14687_amd import window as wn
from test_devices import Stream, calls, there  # noqa: F401


@pytest.fixture
def window_calls(calls, monkeypatch):   # noqa: F811
    wn._library()
    monkeypatch.setattr(wn, "_native", wn._NoNative)
    monkeypatch.setattr(wn, "_lib", sq._lib)   # (the recorder)
    return calls


def entries(stream):
    Q, K, lse = there(1, 4, 64, 64), there(1, 2, 64, 64), there(1, 4, 64, dtype=torch.float32)
    C, S = there(1, 2, 64, 64, dtype=torch.float8_e4m3fn), there(1, 2, 64, dtype=torch.float32)
    table, start, s = there(64, 32, 2, dtype=torch.float32), there(1, dtype=torch.int32), dict(stream=stream)
    eight = dict(K_scale=S, V_scale=S, **s)
    return {
        "grat_window_attention_fwd": lambda: grat.grat_window_attention_fwd(Q, K, K, 0.1, window=5, return_lse=True, **s),
        "grat_window_attention_bwd": lambda: grat.grat_window_attention_bwd(Q, Q, K, K, Q, lse, 0.1, window=5, **s),
        "grat_cache_append": lambda: grat.grat_cache_append(Q, K, K, table, C, C, start, **eight),
        "grat_cache_read": lambda: grat.grat_cache_read(C, S, torch.bfloat16, k_len=start, **s),
        "grat_cache_attention_fwd": lambda: grat.grat_cache_attention_fwd(Q, C, C, 0.1, k_len=start, parent=there(64, dtype=torch.int32), return_lse=True, **eight),
    }


@pytest.mark.parametrize("name", entries(None))
def test_the_tensors_device_is_current(window_calls, name):
    entries(None)[name]()
    assert window_calls == [(name, 1, 101)]


@pytest.mark.parametrize("name", entries(None))
def test_a_stream_of_the_tensors_device(window_calls, name):
    stream = Stream(1)
    stream.cuda_stream = 777
    entries(stream)[name]()
    assert window_calls == [(name, 1, 777)]


@pytest.mark.parametrize("name", entries(None))
def test_a_stream_of_another_device_is_refused(window_calls, name):
    with pytest.raises(ValueError, match="stream"):
        entries(Stream(0))[name]()
    assert not window_calls
