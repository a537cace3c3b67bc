"""What the device found, read without a workspace of the caller's."""
import numpy as np
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import gpu

pytestmark = pytest.mark.gpu
BAD_SEQLENS, BAD_PAGE = 6, 7


@pytest.fixture(autouse=True)
def no_calls_so_far(cuda_lib):
    """Nor any reported by these tests to others, which look at every stream."""
    cuda_lib._stream_ws_cache.clear()
    yield
    cuda_lib._stream_ws_cache.clear()


@pytest.mark.parametrize("R", [1, 150])
def test_every_call_s_status_is_read(cuda_lib, R):
    status = cuda_lib.sa_cache_get_device_error
    cache = cc.Cache([100, 60], 1, 64, 64, seed=61)
    pool, table, lens = cache.tensors()
    cu = gpu(cc.offsets([R, R]))
    q = torch.randn((2 * R, 1, 64), device="cuda").requires_grad_(True)
    gone = table.clone()
    gone[0, 1] = -1
    out = cuda_lib.sa_cache_attention(q, cu, pool, table, lens)
    assert status() == 0
    cuda_lib.sa_cache_attention(q, cu, pool, gone, lens)
    assert status() == BAD_PAGE
    out.sum().backward()  # the next call, in autograd's own thread
    assert status() == 0
    bad = cuda_lib.sa_cache_attention(q, cu, pool, gone, lens)
    status()
    cuda_lib.sa_cache_attn_fwd(q.detach(), cu, pool, table, lens)
    assert status() == 0
    bad.sum().backward()
    assert status() == BAD_PAGE
    cuda_lib.sa_cache_attn_fwd(q.detach(), gpu(np.array([0, 2 * R + 1, 2 * R], np.int32)), pool, table, lens)
    assert status() == BAD_SEQLENS and status("cuda") == BAD_SEQLENS and status(0) == BAD_SEQLENS
    with pytest.raises(cuda_lib.SketchError):  # refused before anything ran: the status stays
        cuda_lib.sa_cache_attn_fwd(q.detach(), cu, pool, table, lens, scale=float("inf"))
    assert status() == BAD_SEQLENS


def test_rows_and_other_streams(cuda_lib):
    status = cuda_lib.sa_cache_get_device_error
    pool = cuda_lib.sa_cache_alloc(4, 1, 64, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    K = torch.randn((160, 1, 64), device="cuda")
    cu = gpu(np.array([0, 100, 160], np.int32))
    late = gpu(np.array([0, 69], np.int32))
    cuda_lib.sa_cache_write(pool, table, K, K, cu)
    assert status() == 0
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        assert status() == 0  # no call yet
        cuda_lib.sa_cache_write(pool, table, K, K, cu, start=late)
        assert status() == BAD_SEQLENS
        cuda_lib.sa_cache_read(pool, table, cu, 160, 64)
        assert status() == 0
        cuda_lib.sa_cache_read(pool, table - 1, cu, 160, 64)
        assert status() == BAD_PAGE
    assert status() == 0


def test_a_caller_s_workspace_has_its_own(cuda_lib):
    cache = cc.Cache([100], 1, 64, 64, seed=62)
    pool, table, lens = cache.tensors()
    cu = gpu(np.array([0, 1], np.int32))
    q = torch.randn((1, 1, 64), device="cuda")
    ws = torch.empty(cuda_lib.sa_cache_attn_workspace_size(1, 1, 1, 1, 64, cuda_lib.SA_F32, 128, False), dtype=torch.uint8,
                     device="cuda")
    cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens)
    cuda_lib.sa_cache_attn_fwd(q, cu, pool, table - 9, lens, ws=ws)
    assert cuda_lib.sa_cache_get_device_error() == 0 and cuda_lib.sa_get_device_error(ws) == BAD_PAGE


def test_a_replay_s_status(cuda_lib):
    cache = cc.Cache([100], 1, 64, 64, seed=63)
    pool, table, lens = cache.tensors()
    cu = gpu(np.array([0, 1], np.int32))
    q = torch.randn((1, 1, 64), device="cuda")
    s, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=s):
        cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens)
    for bad in (False, True, False):
        keep = table.clone()
        if bad:
            table.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            assert cuda_lib.sa_cache_get_device_error() == (BAD_PAGE if bad else 0)
        table.copy_(keep)
