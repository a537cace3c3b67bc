"""Sizes of the linear layers' workspaces (no GPU)."""
import pytest

from paper_2609_08443_gb300 import binding, build

NONE, GELU, SWIGLU = 0, 2, 4
BF16, F32 = 1, 0


@pytest.fixture(scope="module")
def size():
    build.build()
    lib = binding.load()
    return lambda M, N, K, act, dt, bwd, repack=0: lib.sa_linear_workspace_size(M, N, K, act, dt, bwd, repack)


def test_dtype_codes():
    assert (binding.SA_BF16, binding.SA_F32) == (BF16, F32)


@pytest.mark.parametrize("M", [17, 4000, 70001])
def test_an_activation_s_fp32_gradient_is_held_once(size, M):
    """dz goes straight into the terms of the products, whose place a copy of dy's terms takes without an activation."""
    assert size(M, 512, 384, GELU, F32, 1) == size(M, 512, 384, NONE, F32, 1)


@pytest.mark.parametrize("M", [1, 16])
def test_few_rows_hold_dz_as_it_is(size, M):
    """Without the tensor cores there are no terms: 4 bytes an element."""
    assert 0 <= size(M, 512, 384, GELU, F32, 1) - size(M, 512, 384, NONE, F32, 1) - M * 512 * 4 < 256


def test_bf16_holds_dz_or_a_copy_of_dy(size):
    M, N, K = 4000, 512, 384
    plain = size(M, N, K, NONE, BF16, 1)
    assert size(M, N, K, NONE, BF16, 1, 4) - plain == size(M, N, K, GELU, BF16, 1) - plain == M * N * 2


def test_an_unaligned_w_is_copied_above_four_rows(size):
    """bf16 gradients: up to four rows read W where it is, the others from aligned rows."""
    N, K = 512, 333
    for M, copied in ((1, 0), (4, 0), (5, 1), (16, 1), (17, 1)):
        more = size(M, N, K, NONE, BF16, 1, 2) - size(M, N, K, NONE, BF16, 1, 0)
        assert more == copied * (N * 336 * 2), M
