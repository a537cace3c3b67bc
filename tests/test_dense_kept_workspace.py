"""Workspaces that linear layers take for themselves, without a GPU: what is kept between calls."""
import threading

import pytest
import torch

from paper_2609_08443_gb300 import binding


@pytest.fixture
def need(monkeypatch):
    """need(n): later calls want n bytes.  Workspaces are on the host."""
    empty, now = torch.empty, [0]
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw))
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(binding, "_dense_ws_cache", {})
    monkeypatch.setattr(binding, "_dense_ws", threading.local())
    monkeypatch.setattr(binding, "_linear_workspace_size", lambda index, *sizes: now[0])
    return lambda n: now.__setitem__(0, n)


def call(stream=7):
    buf = binding._linear_workspace(None, 0, stream)
    binding._note_call(buf, 0, stream, binding._dense_ws_cache)
    return buf


def held():
    kept = {**binding._dense_ws.__dict__, **{("status", *k): v for k, v in binding._dense_ws_cache.items()}}
    return sum({v.data_ptr(): v.numel() for v in kept.values()}.values())


def test_small_ones_are_kept(need):
    need(1 << 20)
    a = call()
    need(1 << 10)
    assert call().data_ptr() == a.data_ptr()


def test_a_large_one_goes_with_the_next_call(need):
    need(1 << 30)
    assert call().numel() >= 1 << 30 and held() >= 1 << 30  # its status can still be read
    need(4096)
    assert call().numel() >= 4096 and held() <= 1 << 20


def test_a_large_one_is_not_kept_by_each_thread(need):
    need(1 << 30)
    a = call()
    t = threading.Thread(target=call)
    t.start()
    t.join()
    del a
    assert held() < 2 << 30


def test_two_large_ones_are_not_held_at_once(need, monkeypatch):
    need(1 << 30)
    call()
    empty, at = torch.empty, []
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: (at.append(held()), empty(*a, **kw))[1])
    call()
    assert at == [0]
