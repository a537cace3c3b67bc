"""The workspace that a cache call takes for itself, without a GPU: which memory two calls may share."""
import threading

import pytest
import torch

from paper_2609_08443_gb300 import binding


@pytest.fixture
def capturing(monkeypatch):
    """Workspaces on the host, whatever device is asked for; set() says whether the stream is capturing."""
    empty, now = torch.empty, threading.Event()
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", now.is_set)
    monkeypatch.setattr(binding, "_stream_ws_cache", {})
    return now


def apart(a, b):
    return a.data_ptr() + a.numel() <= b.data_ptr() or b.data_ptr() + b.numel() <= a.data_ptr()


def in_a_thread(f):
    got = []
    t = threading.Thread(target=lambda: got.append(f()))
    t.start()
    t.join()
    return got[0]


def test_two_threads_calls_on_one_stream_share_nothing(capturing):
    """Each may be between the two launches of its call."""
    a = binding._stream_workspace(4096, 0, 7001)
    assert apart(a, in_a_thread(lambda: binding._stream_workspace(1024, 0, 7001)))


def test_a_captured_call_shares_nothing_with_the_stream_s_others(capturing):
    before = binding._stream_workspace(4096, 0, 7002)
    capturing.set()
    a, b = (binding._stream_workspace(4096, 0, 7002) for _ in range(2))
    capturing.clear()
    after = binding._stream_workspace(4096, 0, 7002)
    assert apart(a, b) and all(apart(x, y) for x in (a, b) for y in (before, after))
    # nor is the first call of a stream, captured, what its later ones get
    capturing.set()
    a = binding._stream_workspace(4096, 0, 7003)
    capturing.clear()
    assert apart(a, binding._stream_workspace(4096, 0, 7003))


def test_few_streams_keep_a_buffer(capturing):
    for stream in range(8000, 9000):
        binding._stream_workspace(64, 0, stream)
    assert len(binding._stream_ws_cache) <= 16

    def after_many():
        for stream in range(8000, 9000):
            binding._stream_workspace(64, 0, stream)
        return len(binding._own_ws.__dict__)

    assert in_a_thread(after_many) <= 16


def test_a_size_is_remembered_for_the_device_it_holds_on(monkeypatch):
    """It follows the current device's SM count."""
    class Library:
        def sa_cache_attn_workspace_size(self, *sizes):
            return 1000 + device

    monkeypatch.setattr(binding, "load", Library)
    sizes = []
    for device in (0, 1, 0):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
        sizes.append(binding.sa_cache_attn_workspace_size(7001, 3, 2, 1, 64, 1, 128, False))
    assert sizes == [1000, 1001, 1000]
    binding._attn_workspace_size.cache_clear()
    device = 0
    assert binding._attn_workspace_size(0, 7001, 3, 2, 1, 64, 1, 128, 0) == 1000
    device = 1
    assert binding._attn_workspace_size(1, 7001, 3, 2, 1, 64, 1, 128, 0) == 1001
    binding._attn_workspace_size.cache_clear()
