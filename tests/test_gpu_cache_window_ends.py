"""Windows whose ends are far outside the cache, down to the type's lowest and up to its highest value."""
import numpy as np
import pytest

import cache_cases as cc
from test_gpu_cache import run_both

pytestmark = pytest.mark.gpu
LOW, HIGH = -(1 << 31), (1 << 31) - 1
ENDS = [(0, LOW), (LOW, LOW), (HIGH, HIGH), (HIGH, LOW), (LOW, HIGH), (0, HIGH), (LOW, 0), (300, LOW + 300), (HIGH, 0), (100, 250)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("R", [1, 10, 160, 300])
def test_far_ends(cuda_lib, dt, d, R):
    cache = cc.Cache([700, 0, 129], 1, d, 64, seed=71)
    for turn in range(len(ENDS) if R == 1 else 1):
        begin, end = (np.array([ENDS[(i + turn) % len(ENDS)][k] for i in range(3 * R)]) for k in range(2))
        run_both(cuda_lib, cache, [R] * 3, 1, dt, begin=begin, end=end)
