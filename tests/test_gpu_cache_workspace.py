"""Calls without a workspace of the caller's: captured in graphs, from two threads, beside each other."""
import threading

import numpy as np
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import gpu

pytestmark = pytest.mark.gpu


class Calls:
    """Forward and gradient of R queries each of some users."""

    def __init__(self, lib, lens, R, seed):
        cache = cc.Cache(lens, 2, 128, 64, seed=seed)
        self.lib, self.cache = lib, cache.tensors()
        self.cu = gpu(cc.offsets([R] * len(lens)))
        self.q, self.do = (torch.randn((R * len(lens), 2, 128), device="cuda").bfloat16() for _ in range(2))

    def __call__(self):
        out, lse = self.lib.sa_cache_attn_fwd(self.q, self.cu, *self.cache, want_lse=True)
        return out, lse, self.lib.sa_cache_attn_bwd(self.q, self.cu, *self.cache, out, lse, self.do)


def equal(x, y):
    return all(torch.equal(a, b) for a, b in zip(x, y))


@pytest.mark.parametrize("R", [1, 150])
def test_a_graph_s_workspace_is_its_own(cuda_lib, R):
    small = Calls(cuda_lib, [3000, 10, 700], R, 51)
    large = Calls(cuda_lib, [9000] * 4, 300, 52)
    ref, ref_large = small(), large()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):  # the stream's first call: nothing is there beforehand
            got = small()
        assert equal(large(), ref_large)
    torch.cuda.synchronize()
    # whatever the allocator may give away now holds a pattern
    taken = [torch.full((1 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(100)]
    with torch.cuda.stream(s):
        taken += [torch.full((8 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(10)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x in got:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert equal(got, ref)
        assert all(bool((x == 0x5A).all()) for x in taken)


@pytest.mark.parametrize("R", [1, 150])
def test_replays_beside_eager_calls_on_the_capture_stream(cuda_lib, R):
    small = Calls(cuda_lib, [6000, 10, 700], R, 53)
    other = Calls(cuda_lib, [2000, 4000, 30, 5000], R, 54)
    ref, ref_other = small(), other()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        got = small()
    for _ in range(50):
        graph.replay()  # on the default stream
        with torch.cuda.stream(s):
            eager = other()
        torch.cuda.synchronize()
        assert equal(got, ref) and equal(eager, ref_other)


def test_two_threads_on_one_stream(cuda_lib):
    calls = [Calls(cuda_lib, [3000, 10, 700], 1, 55), Calls(cuda_lib, [2000] * 5, 150, 56), Calls(cuda_lib, [900], 3, 57)]
    refs = [c() for c in calls]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        got = [calls[i]() for _ in range(200)]
        torch.cuda.synchronize()
        wrong.append(sum(not equal(g, refs[i]) for g in got))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(3)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert wrong == [0, 0, 0]


def test_rows_in_a_graph(cuda_lib):
    pool = cuda_lib.sa_cache_alloc(4, 2, 64, 64)
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(2, 2)
    cu = gpu(np.array([0, 100, 190], np.int32))
    K = torch.randn((190, 2, 64), device="cuda").bfloat16()
    cuda_lib.sa_cache_write(pool, table, K, -K, cu)
    k, v = cuda_lib.sa_cache_read(pool, table, cu, 190, 64)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cuda_lib.sa_cache_write(pool, table, K, -K, cu)
        kg, vg = cuda_lib.sa_cache_read(pool, table, cu, 190, 64)
    pool.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(kg, k) and torch.equal(vg, v)
