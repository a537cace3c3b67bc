"""The cache's C entry points exist, and what the host can refuse it refuses without a GPU."""
import ctypes
import os
import re

import pytest

from paper_2609_08443_gb300 import binding, build

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "sa_cache.h")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(sa_cache_[a-z_]+)\s*\(", text))
    assert len(names) == 7
    for name in names:
        assert hasattr(lib, name), name


def test_status_string(lib):
    assert "block_table" in binding.sa_status_string(7)


def test_page_bytes(lib):
    assert binding.sa_cache_page_bytes(8, 128, 64) == 8 * 2 * 64 * 72
    for H, d, page in ((0, 64, 64), (65, 64, 64), (1, 8, 64), (1, 136, 64), (1, 24, 64), (1, 64, 8), (1, 64, 48),
                       (1, 64, 512)):
        assert binding.sa_cache_page_bytes(H, d, page) == 0


def vp(x):
    return ctypes.c_void_p(x) if x else None


def write(lib, **kw):
    a = dict(K=4096, V=4096, us=0, rs=128, hs=64, cu=4096, B=2, N=4, start=0, H=2, d=64, dt=1, pool=4096, n_pages=4,
             page=64, table=4096, max_pages=2, ws=4096, wsb=256)
    a.update(kw)
    return lib.sa_cache_write(vp(a["K"]), vp(a["V"]), a["us"], a["rs"], a["hs"], vp(a["cu"]), a["B"], a["N"],
                              vp(a["start"]), a["H"], a["d"], a["dt"], vp(a["pool"]), a["n_pages"], a["page"],
                              vp(a["table"]), a["max_pages"], vp(a["ws"]), a["wsb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(K=0), INVALID), (dict(V=4098), INVALID), (dict(pool=0), INVALID), (dict(pool=4104), INVALID),
    (dict(table=0), INVALID), (dict(B=0), INVALID), (dict(N=-1), INVALID), (dict(rs=129), INVALID),
    (dict(hs=4), INVALID), (dict(hs=-64), INVALID), (dict(cu=0, N=5), INVALID), (dict(ws=0), INVALID),
    (dict(ws=4104), INVALID), (dict(n_pages=0), INVALID), (dict(max_pages=0), INVALID),
    (dict(page=48), UNSUPPORTED), (dict(page=8), UNSUPPORTED), (dict(d=40), UNSUPPORTED), (dict(d=144), UNSUPPORTED),
    (dict(H=65), UNSUPPORTED), (dict(dt=2), UNSUPPORTED), (dict(N=1 << 31), UNSUPPORTED),
    (dict(max_pages=1 << 30), UNSUPPORTED), (dict(wsb=128), WORKSPACE)])
def test_write_refuses(lib, kw, want):
    assert write(lib, **kw) == want


def attn(lib, bwd=False, **kw):
    a = dict(q=4096, qr=256, qh=64, cu=4096, B=2, T=4, Hq=4, pool=4096, n_pages=4, page=64, table=4096, max_pages=2,
             lens=4096, H=2, d=64, scale=0.125, dt=1, out=4096, lse=4096, dout=4096, dq=4096, ws=4096, wsb=1 << 40)
    a.update(kw)
    head = (vp(a["q"]), a["qr"], a["qh"], vp(a["cu"]), a["B"], a["T"], a["Hq"], vp(a["pool"]), a["n_pages"], a["page"],
            vp(a["table"]), a["max_pages"], vp(a["lens"]), a["H"], a["d"], None, None, a["scale"], a["dt"])
    if bwd:
        return lib.sa_cache_attn_bwd(*head, vp(a["out"]), vp(a["lse"]), vp(a["dout"]), vp(a["dq"]), vp(a["ws"]),
                                     a["wsb"], None)
    return lib.sa_cache_attn_fwd(*head, vp(a["out"]), vp(a["lse"]), vp(a["ws"]), a["wsb"], None)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,want", [
    (dict(q=0), INVALID), (dict(q=4100), INVALID), (dict(cu=0), INVALID), (dict(lens=0), INVALID),
    (dict(out=0), INVALID), (dict(out=4104), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(scale=float("nan")), INVALID), (dict(qr=100), INVALID), (dict(qh=-8), INVALID), (dict(T=-1), INVALID),
    (dict(B=0), INVALID), (dict(Hq=0), INVALID), (dict(Hq=3), UNSUPPORTED), (dict(Hq=1), UNSUPPORTED),
    (dict(d=72), UNSUPPORTED), (dict(dt=5), UNSUPPORTED), (dict(page=100), UNSUPPORTED),
    (dict(T=1 << 31), UNSUPPORTED), (dict(wsb=1024), WORKSPACE), (dict(ws=4096 + 64), INVALID)])
def test_attention_refuses(lib, bwd, kw, want):
    assert attn(lib, bwd, **kw) == want


@pytest.mark.parametrize("kw", [dict(lse=0), dict(dout=0), dict(dq=0), dict(dq=4104)])
def test_gradient_refuses(lib, kw):
    assert attn(lib, True, **kw) == INVALID


def test_workspace_size_rejects_bad_sizes(lib):
    size = binding.sa_cache_attn_workspace_size
    assert size(2, 4, 4, 2, 64, 1, 128, False) > 0
    for a in ((0, 4, 4, 2, 64, 1, 128), (2, -1, 4, 2, 64, 1, 128), (2, 4, 3, 2, 64, 1, 128), (2, 4, 4, 2, 20, 1, 128),
              (2, 4, 4, 2, 64, 9, 128), (2, 4, 4, 2, 64, 1, -1)):
        assert size(*a, False) == 0
