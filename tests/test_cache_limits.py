"""Sizes whose tiles would pass 32-bit indexes are refused: the kernels count a user's positions and rows in
int32 and round both up to a tile (at most 256)."""
import pytest

from paper_2609_08443_gb300 import binding
from test_cache_abi import INVALID, UNSUPPORTED, attn, lib, write  # noqa: F401

MOST = (1 << 31) - 256


@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("bwd", [False, True])
def test_positions(lib, page, bwd):  # noqa: F811
    last = MOST // page
    assert attn(lib, bwd, page=page, max_pages=last + 1) == UNSUPPORTED
    assert attn(lib, bwd, page=page, max_pages=last, ws=0) == INVALID  # looked at after the sizes


@pytest.mark.parametrize("page", [16, 64, 256])
def test_rows_written(lib, page):  # noqa: F811
    assert write(lib, page=page, max_pages=MOST // page + 1) == UNSUPPORTED
    assert write(lib, page=page, max_pages=MOST // page, ws=0) == INVALID


@pytest.mark.parametrize("Hq", [2, 4, 10])
@pytest.mark.parametrize("bwd", [False, True])
def test_query_rows_of_a_cached_head(lib, Hq, bwd):  # noqa: F811
    G = Hq // 2
    last = MOST // G
    assert attn(lib, bwd, Hq=Hq, T=last + 1) == UNSUPPORTED
    assert attn(lib, bwd, Hq=Hq, T=last, ws=0) == INVALID
    size = binding.sa_cache_attn_workspace_size
    assert size(2, last + 1, Hq, 2, 64, 1, 128, bwd) == 0 and size(2, last, Hq, 2, 64, 1, 128, bwd) > 0
