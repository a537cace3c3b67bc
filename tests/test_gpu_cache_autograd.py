"""What autograd has to refuse: a gradient over pages that were rewritten, and a second derivative."""
import numpy as np
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import gpu

pytestmark = pytest.mark.gpu


def setup(L=100, R=3):
    cache = cc.Cache([L], 1, 64, 64, seed=31)
    pool, table, lens = cache.tensors()
    q = torch.randn((R, 1, 64), device="cuda").requires_grad_(True)
    return pool, table, lens, gpu(np.array([0, R], np.int32)), q


def rows(n):
    return torch.randn((n, 1, 64), device="cuda"), gpu(np.array([0, n], np.int32))


def test_rows_rewritten_before_the_backward_are_refused(cuda_lib):
    pool, table, lens, cu, q = setup()
    out = cuda_lib.sa_cache_attention(q, cu, pool, table, lens)
    K, n = rows(10)
    cuda_lib.sa_cache_write(pool, table, K, K, n)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_a_page_given_to_somebody_else_is_refused(cuda_lib):
    cache = cc.Cache([100, 60], 1, 64, 64, seed=32)
    pool, table, lens = cache.tensors()
    q = torch.randn((2, 1, 64), device="cuda").requires_grad_(True)
    out = cuda_lib.sa_cache_attention(q, gpu(np.array([0, 1, 2], np.int32)), pool, table, lens)
    K, n = rows(60)
    cuda_lib.sa_cache_write(pool, table[1:].contiguous(), K, K, n)  # the second user's page gets other rows
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_appended_rows_may_be_declared(cuda_lib):
    pool, table, lens, cu, q = setup(L=100)
    cuda_lib.sa_cache_attention(q, cu, pool, table, lens).sum().backward()
    want, q.grad = q.grad, None
    out = cuda_lib.sa_cache_attention(q, cu, pool, table, lens)
    K, n = rows(20)
    cuda_lib.sa_cache_write(pool, table, K, K, n, start=lens, appends=True)
    out.sum().backward()
    assert torch.equal(q.grad, want)


def test_a_write_before_the_forward_changes_nothing(cuda_lib):
    pool, table, lens, cu, q = setup(L=100)
    K, n = rows(10)
    cuda_lib.sa_cache_write(pool, table, K, K, n)
    cuda_lib.sa_cache_attention(q, cu, pool, table, lens).sum().backward()
    assert torch.isfinite(q.grad).all()
    with torch.inference_mode():
        cuda_lib.sa_cache_write(pool, table, K, K, n)


def test_a_second_derivative_is_refused(cuda_lib):
    pool, table, lens, cu, q = setup()
    out = cuda_lib.sa_cache_attention(q, cu, pool, table, lens)
    dq, = torch.autograd.grad(out.square().sum(), q, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        dq.sum().backward()
