"""Positions between the windows of a user's queries that no query sees: never written, without a page, or
holding bytes that no written row has."""
import numpy as np
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import gpu, run_both

pytestmark = pytest.mark.gpu

# (code byte, scale byte): NaN and infinity as float16, scales past the largest, level -8 times the largest two
BYTES = [(0xFF, 0xFF), (0x88, 0xFF), (0x00, 0xF8), (0x00, 0xE2), (0x00, 0xE1), (0x00, 0xE0)]


def windows(L, R):
    """Queries see the first few or the last few rows, in turn."""
    i = np.arange(R)
    begin = np.where(i % 2 == 0, 0, L - 50 + i % 7)
    end = np.where(i % 2 == 0, 10 + i % 3, L - i % 5)
    return begin, end


def fill(cache, lo, hi, code, scale):
    """Positions lo .. hi - 1 of user 0 get these bytes."""
    page, d = cache.page, cache.d
    for p in range(lo // page, -(-hi // page)):
        a, b = max(lo - p * page, 0), min(hi - p * page, page)
        rec = cache.pool[cache.table[0, p]]
        rec[..., a * d // 2: b * d // 2] = code
        rec[..., page * d // 2 + a * d // 16: page * d // 2 + b * d // 16] = scale


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16), (128, 64), (128, 256), (96, 32)])
@pytest.mark.parametrize("R,L", [(2, 500), (13, 500), (160, 500), (300, 500), (2, 6000), (160, 6000)])
def test_bytes_between_the_windows_never_matter(cuda_lib, dt, d, page, R, L):
    cache = cc.Cache([L], 1, d, page, seed=21)
    begin, end = windows(L, R)
    base = run_both(cuda_lib, cache, [R], 1, dt, begin=begin, end=end)
    for code, scale in BYTES:
        fill(cache, 12, L - 50, code, scale)
        got = run_both(cuda_lib, cache, [R], 1, dt, begin=begin, end=end)
        for a, b in zip(base, got):
            assert torch.equal(a, b), (code, scale)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,page", [(64, 64), (128, 16), (128, 64), (128, 256), (96, 32)])
@pytest.mark.parametrize("R,L", [(2, 700), (13, 700), (160, 700), (2, 6000), (160, 6000)])
def test_pages_between_the_windows_may_be_missing(cuda_lib, dt, d, page, R, L):
    """run_both asserts that the call reported nothing."""
    cache = cc.Cache([L], 1, d, page, seed=22)
    begin, end = windows(L, R)
    base = run_both(cuda_lib, cache, [R], 1, dt, begin=begin, end=end)
    first, last = -(-12 // page), (L - 50) // page  # whole pages that nobody sees
    assert first < last
    for gone in (-1, cache.n_pages):
        cache.table[0, first:last] = gone
        got = run_both(cuda_lib, cache, [R], 1, dt, begin=begin, end=end)
        for a, b in zip(base, got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R", [3, 160])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_a_missing_page_that_one_query_sees_is_reported(cuda_lib, dt, R, page):
    cache = cc.Cache([700], 1, 128, page, seed=23)
    begin, end = windows(700, R)
    begin[R // 2], end[R // 2] = 300, 301
    cache.table[0, 300 // page] = -1
    pool, table, lens = cache.tensors()
    cu = gpu(cc.offsets([R]))
    q = cc.to_gpu(cc.queries(R, 1, 128, dt, 1), dt)
    kw = {"kv_begin": gpu(begin.astype(np.int32)), "kv_end": gpu(end.astype(np.int32))}
    size = [cuda_lib.sa_cache_attn_workspace_size(1, R, 1, 1, 128, cuda_lib.SA_BF16 if dt == "bf16" else cuda_lib.SA_F32,
                                                  700, bwd) for bwd in (False, True)]
    ws = torch.empty(max(size), dtype=torch.uint8, device="cuda")
    out, lse = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, want_lse=True, ws=ws, **kw)
    assert cuda_lib.sa_get_device_error(ws) == 7
    cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, out, lse, q, ws=ws, **kw)
    assert cuda_lib.sa_get_device_error(ws) == 7


@pytest.mark.parametrize("entry", [-1, -2, -3, -(1 << 31), 3, (1 << 31) - 1])
@pytest.mark.parametrize("R", [3, 160])
@pytest.mark.parametrize("bwd", [False, True])
def test_every_entry_outside_the_pool_is_reported(cuda_lib, entry, R, bwd):
    cache = cc.Cache([130], 1, 64, 64, seed=25, spare=0)
    assert cache.n_pages == 3
    cache.table[0, 1] = entry
    pool, table, lens = cache.tensors()
    cu = gpu(cc.offsets([R]))
    q = cc.to_gpu(cc.queries(R, 1, 64, "bf16", 1), "bf16")
    ws = torch.empty(cuda_lib.sa_cache_attn_workspace_size(1, R, 1, 1, 64, cuda_lib.SA_BF16, 130, bwd), dtype=torch.uint8,
                     device="cuda")
    if bwd:
        lse = torch.zeros((R, 1), device="cuda")
        cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, q, lse, q, ws=ws)
    else:
        cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, ws=ws)
    assert cuda_lib.sa_get_device_error(ws) == 7


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,R", [(64, 3), (128, 3), (64, 160), (128, 160)])
def test_values_near_the_largest_in_partly_hidden_blocks(cuda_lib, dt, d, R):
    """The scales 8192 and 9216, whose level -8 no float16 holds, are values like any other where they were written."""
    cache = cc.Cache([300], 1, d, 64, seed=24, v_std=4e4)
    begin, end = windows(300, R)
    end[::3] = 150
    run_both(cuda_lib, cache, [R], 1, dt, begin=begin, end=end)
