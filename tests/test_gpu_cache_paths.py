"""sa_select_path: the cache's attention on its warp-level kernels where the tcgen05 ones would be taken."""
import pytest
import torch

import cache_cases as cc
from test_gpu_cache import run_both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_both_kernels_answer_the_same_call(cuda_lib, d):
    cache = cc.Cache([300, 77, 512], 1, d, 64, seed=41)
    names, got = [], []
    try:
        for path in (0, 1):
            cuda_lib.sa_select_path(path)
            names += [cuda_lib.sa_cache_attn_kernel_name(3, 450, 1, 1, d, 0.1, cuda_lib.SA_BF16, bwd) for bwd in (False, True)]
            got.append(run_both(cuda_lib, cache, [150] * 3, 1, "bf16", seed=41))
    finally:
        cuda_lib.sa_select_path(0)
    assert [n[:3] for n in names] == ["tc5", "tc5", "mma", "mma"]
    # each is within its bounds of the oracle (run_both); lse has no roundings to 16 bits
    assert torch.allclose(got[0][1], got[1][1], atol=1e-4)


def test_a_workspace_serves_every_path(cuda_lib):
    """Its size does not follow the switch: a buffer sized under one path is used under another."""
    sizes = []
    try:
        for path in (0, 1, 2, 3):
            cuda_lib.sa_select_path(path)
            sizes += [[cuda_lib.load().sa_cache_attn_workspace_size(3, 450, 1, 1, 128, 1, 512, bwd) for bwd in (0, 1)]]
    finally:
        cuda_lib.sa_select_path(0)
    assert all(s == sizes[0] for s in sizes) and min(sizes[0]) > 0
