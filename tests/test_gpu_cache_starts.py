"""A start that the device finds out of range: the call writes nothing, whichever user it belongs to."""
import numpy as np
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import gpu

pytestmark = pytest.mark.gpu

STARTS = [[-1, 0, 0], [0, 0, -(1 << 31)], [0, 69, 0], [0, 0, 129], [1 << 30, 0, 0], [0, (1 << 31) - 1, 0]]


@pytest.mark.parametrize("start", STARTS)
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_a_bad_start_writes_nothing(cuda_lib, start, dt):
    H, d, page = 2, 64, 64
    pool = cuda_lib.sa_cache_alloc(6, H, d, page)
    pool.random_(0, 256)
    before = pool.clone()
    table = torch.arange(6, dtype=torch.int32, device="cuda").view(3, 2)
    w = torch.empty(256, dtype=torch.uint8, device="cuda")
    first = gpu(np.array(start, np.int32))
    K = torch.randn((180, H, d), device="cuda").to(cc.TORCH[dt])
    cu = gpu(np.array([0, 60, 120, 180], np.int32))
    cuda_lib.sa_cache_write(pool, table, K, K, cu, start=first, ws=w)  # packed rows
    assert cuda_lib.sa_get_device_error(w) == 6 and torch.equal(pool, before)
    S = torch.randn((3, H, 60, d), device="cuda").to(cc.TORCH[dt])
    cuda_lib.sa_cache_write(pool, table, S, S, start=first, ws=w)  # equal counts
    assert cuda_lib.sa_get_device_error(w) == 6 and torch.equal(pool, before)
    cuda_lib.sa_cache_read(pool, table, cu, 180, d, start=first, ws=w)
    assert cuda_lib.sa_get_device_error(w) == 6
    good = gpu(np.array([0, 68, 3], np.int32))
    cuda_lib.sa_cache_write(pool, table, K, K, cu, start=good, ws=w)
    assert cuda_lib.sa_get_device_error(w) == 0 and not torch.equal(pool, before)


def test_equal_counts_that_pass_the_table_write_nothing(cuda_lib):
    pool = cuda_lib.sa_cache_alloc(4, 1, 64, 64)
    pool.random_(0, 256)
    before = pool.clone()
    table = torch.arange(4, dtype=torch.int32, device="cuda").view(4, 1)
    w = torch.empty(256, dtype=torch.uint8, device="cuda")
    S = torch.randn((4, 1, 65, 64), device="cuda")
    cuda_lib.sa_cache_write(pool, table, S, S, ws=w)
    assert cuda_lib.sa_get_device_error(w) == 6 and torch.equal(pool, before)
