"""The 4-bit cache's fp64 reference, pinned by brute force, exactness and finite differences."""
import numpy as np
import pytest

from oracle import cache_oracle as co


def brute(x):
    """One group: every scale tried in order, every level tried."""
    big = np.max(np.abs(x))
    code = next((int(c) for c, s in zip(co.CODES, co.SCALES) if 7.5 * s >= big), int(co.CODES[-1]))
    s = (8 + code % 8) * 2.0 ** (code // 8 - 18)
    out = []
    for v in x:
        best = min(range(-7, 8), key=lambda l: (abs(v - l * s), abs(l)))
        out.append(best)
    return np.array(out), code


@pytest.mark.parametrize("std", [1e-6, 1e-4, 0.02, 1.0, 300.0, 2e4, 1e6])
def test_groups_against_brute_force(std):
    rng = np.random.default_rng(5)
    for _ in range(20):
        x = (rng.standard_normal(16) * std).astype(np.float32).astype(np.float64)
        level, code = co.quantise(x)
        want, c = brute(x)
        assert code[0] == c
        assert np.array_equal(level, want)


def test_scales_are_float16_values_and_products_are_exact_in_16_bits():
    f16 = (co.CODES.astype(np.uint16) << 7).view(np.float16).astype(np.float64)
    assert np.array_equal(f16, co.SCALES)
    prod = np.arange(-7, 8)[:, None] * co.SCALES
    assert np.array_equal(prod.astype(np.float16).astype(np.float64), prod)
    bits = prod.astype(np.float32).view(np.uint32)
    assert np.all(bits & 0xFFFF == 0)  # bf16 holds them too


def test_ties_go_to_zero_and_largest_values_saturate():
    x = np.zeros(16)
    x[0], x[1], x[2] = 7.0, 2.5, -2.5  # 7.5 x 15/16 = 7.03 is enough: s = 15/16
    level, code = co.quantise(x)
    assert co.SCALES[code[0] - 8] == 0.9375 and list(level[:3]) == [7, 3, -3]
    x[0] = 7.5  # s = 1
    level, code = co.quantise(x)
    assert co.SCALES[code[0] - 8] == 1.0 and list(level[:3]) == [7, 2, -2]
    assert np.max(np.abs(co.stored(np.full(16, np.inf)))) == 64512.0
    assert not np.any(co.stored(np.full(16, np.nan)))


def test_relative_error_of_a_group():
    x = np.random.default_rng(0).standard_normal((4000, 64))
    e = np.abs(co.stored(x) - x).reshape(-1, 16)
    big = np.abs(x).reshape(-1, 16).max(-1, keepdims=True)
    assert np.all(e <= big / 7.5 * 1.125 / 2 + 1e-12)  # half a step; a step is at most 1.125/7.5 of the largest


def test_record_layout():
    x = np.random.default_rng(1).standard_normal((16, 48))
    rec = co.record(x)
    assert rec.size == 16 * (24 + 3)
    level, code = co.quantise(x)
    word = rec[: 16 * 24].reshape(16, 6, 4).astype(np.uint32)
    word = word[..., 0] | word[..., 1] << 8 | word[..., 2] << 16 | word[..., 3] << 24
    lo, hi = word & 0xFFFF, word >> 16
    for i in range(4):  # the pair (2i, 2i + 1) sits at the same place of the two halves
        assert np.array_equal(((lo >> (4 * i)) & 15).astype(int) - 8, level.reshape(16, 6, 8)[..., 2 * i])
        assert np.array_equal(((hi >> (4 * i)) & 15).astype(int) - 8, level.reshape(16, 6, 8)[..., 2 * i + 1])
    assert np.array_equal(rec[16 * 24:].reshape(16, 3), code)


def test_gradient_against_differences():
    rng = np.random.default_rng(2)
    q, k, v, g = (rng.standard_normal(s) for s in ((5, 16), (23, 16), (23, 16), (5, 16)))
    win = [(0, 23), (4, 9), (7, 7), (22, 23), (0, 1)]
    out, lse = co.attention(q, k, v, 0.3, win)
    dq = co.attention_grad(q, k, v, 0.3, win, out, lse, g)
    assert not out[2].any() and lse[2] == -np.inf and not dq[2].any()
    h = 1e-6
    for r in range(5):
        for c in range(16):
            a, b = q.copy(), q.copy()
            a[r, c] += h
            b[r, c] -= h
            diff = np.sum(g * (co.attention(a, k, v, 0.3, win)[0] - co.attention(b, k, v, 0.3, win)[0])) / (2 * h)
            assert abs(diff - dq[r, c]) < 1e-8
