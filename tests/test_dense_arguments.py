"""What the dense operators refuse, without a GPU: the C entry points' checks and the binding's."""
import ctypes
import os
import re

import pytest
import torch

from paper_2609_08443_gb300 import binding, build

HEADER = os.path.join(os.path.dirname(os.path.dirname(__file__)), "include", "sa_dense.h")
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load()


def vp(x):
    return ctypes.c_void_p(x) if x else None


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(sa_(?:layer_norm|linear)_[a-z_]+)\s*\(", text))
    assert len(names) == 7
    for name in names:
        assert hasattr(lib, name), name


def norm_fwd(lib, **kw):
    a = dict(x=4096, xs=64, xd=1, r=0, rs=0, rd=0, w=4096, b=4096, wd=1, rows=4, n=64, eps=1e-5, y=4096, yd=1, st=0)
    a.update(kw)
    return lib.sa_layer_norm_fwd(vp(a["x"]), a["xs"], a["xd"], vp(a["r"]), a["rs"], a["rd"], vp(a["w"]), vp(a["b"]),
                                 a["wd"], a["rows"], a["n"], a["eps"], vp(a["y"]), a["yd"], vp(a["st"]), None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=0), INVALID), (dict(x=4097), INVALID), (dict(xs=-1), INVALID), (dict(rows=-1), INVALID),
    (dict(n=0), INVALID), (dict(eps=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(y=0), INVALID), (dict(y=4098, yd=0), INVALID), (dict(w=4097), INVALID),
    (dict(b=4097), INVALID), (dict(st=4100), INVALID), (dict(r=4097, rd=1), INVALID), (dict(r=4096, rs=-2), INVALID),
    (dict(xd=2), UNSUPPORTED), (dict(yd=3), UNSUPPORTED), (dict(wd=-1), UNSUPPORTED), (dict(r=4096, rd=7), UNSUPPORTED),
    (dict(n=16385), UNSUPPORTED), (dict(rows=1 << 31), UNSUPPORTED), (dict(rows=0, x=0, y=0), OK)])
def test_norm_forward_refuses(lib, kw, want):
    assert norm_fwd(lib, **kw) == want


def norm_bwd(lib, **kw):
    a = dict(dy=4096, ys=64, yd=1, x=4096, xs=64, xd=1, r=0, rs=0, rd=0, w=4096, wd=1, st=4096, rows=4, n=64, dx=4096,
             dr=0, dw=4096, db=4096, ws=4096, wsb=BIG)
    a.update(kw)
    return lib.sa_layer_norm_bwd(vp(a["dy"]), a["ys"], a["yd"], vp(a["x"]), a["xs"], a["xd"], vp(a["r"]), a["rs"],
                                 a["rd"], vp(a["w"]), a["wd"], vp(a["st"]), a["rows"], a["n"], vp(a["dx"]),
                                 vp(a["dr"]), vp(a["dw"]), vp(a["db"]), vp(a["ws"]), a["wsb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(dy=0), INVALID), (dict(ys=-1), INVALID), (dict(x=0), INVALID), (dict(st=0), INVALID), (dict(st=4100), INVALID),
    (dict(dr=4096), INVALID), (dict(dx=4097), INVALID), (dict(dw=4097), INVALID), (dict(ws=0), INVALID),
    (dict(ws=4100), INVALID), (dict(wsb=256), WORKSPACE), (dict(yd=5), UNSUPPORTED), (dict(n=16385), UNSUPPORTED),
    (dict(dw=0, db=0, dx=0, ws=0), OK), (dict(rows=0, dw=0, db=0, ws=0, x=0, dy=0, st=0), OK)])
def test_norm_backward_refuses(lib, kw, want):
    assert norm_bwd(lib, **kw) == want


def test_sizes(lib):
    assert lib.sa_layer_norm_workspace_size(10, 64) >= 256 + 2 * 64 * 4
    assert lib.sa_layer_norm_workspace_size(10, 16385) == 0 and lib.sa_layer_norm_workspace_size(-1, 64) == 0
    assert lib.sa_linear_workspace_size(10, 64, 64, 0, 1, 0, 7) >= 256
    for bad in ((-1, 64, 64, 0, 1), (1, 0, 64, 0, 1), (1, 64, 0, 0, 1), (1, 64, 64, 5, 1), (1, 64, 64, 0, 2),
                (1 << 31, 64, 64, 0, 1), (1, (1 << 20) + 1, 64, 0, 1), (1, (1 << 19) + 1, 64, 4, 1)):
        assert lib.sa_linear_workspace_size(*bad, 0, 0) == 0


def linear_fwd(lib, **kw):
    a = dict(x=4096, xs=64, w=4096, wst=64, b=0, r=0, rs=0, M=4, N=32, K=64, act=0, dt=1, y=4096, z=0, ws=4096, wsb=BIG)
    a.update(kw)
    return lib.sa_linear_fwd(vp(a["x"]), a["xs"], vp(a["w"]), a["wst"], vp(a["b"]), vp(a["r"]), a["rs"], a["M"],
                             a["N"], a["K"], a["act"], a["dt"], vp(a["y"]), vp(a["z"]), vp(a["ws"]), a["wsb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(x=0), INVALID), (dict(x=4097), INVALID), (dict(w=0), INVALID), (dict(xs=-8), INVALID), (dict(wst=-1), INVALID),
    (dict(r=4097), INVALID), (dict(r=4096, rs=-1), INVALID), (dict(y=0), INVALID), (dict(y=4097), INVALID),
    (dict(z=4097), INVALID), (dict(b=4097), INVALID), (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID),
    (dict(act=-1), INVALID), (dict(act=5), INVALID), (dict(ws=0), INVALID), (dict(ws=4100), INVALID),
    (dict(dt=2), UNSUPPORTED), (dict(M=1 << 31), UNSUPPORTED), (dict(K=(1 << 20) + 1), UNSUPPORTED),
    (dict(N=(1 << 20) + 1), UNSUPPORTED), (dict(wsb=128), WORKSPACE)])
def test_linear_forward_refuses(lib, kw, want):
    assert linear_fwd(lib, **kw) == want


def linear_bwd(lib, **kw):
    a = dict(dy=4096, ys=32, x=4096, xs=64, w=4096, wst=64, z=4096, M=4, N=32, K=64, act=2, dt=1, dx=4096, dw=4096,
             db=4096, ws=4096, wsb=BIG)
    a.update(kw)
    return lib.sa_linear_bwd(vp(a["dy"]), a["ys"], vp(a["x"]), a["xs"], vp(a["w"]), a["wst"], vp(a["z"]), a["M"],
                             a["N"], a["K"], a["act"], a["dt"], vp(a["dx"]), vp(a["dw"]), vp(a["db"]), vp(a["ws"]),
                             a["wsb"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(dy=0), INVALID), (dict(dy=4097), INVALID), (dict(ys=-1), INVALID), (dict(x=0), INVALID), (dict(w=0), INVALID),
    (dict(z=0), INVALID), (dict(z=4097), INVALID), (dict(dx=4097), INVALID), (dict(dw=4097), INVALID),
    (dict(db=4097), INVALID), (dict(ws=0), INVALID), (dict(act=9), INVALID), (dict(dt=5), UNSUPPORTED),
    (dict(M=1 << 31), UNSUPPORTED), (dict(wsb=256), WORKSPACE)])
def test_linear_backward_refuses(lib, kw, want):
    assert linear_bwd(lib, **kw) == want


def test_kernel_names(lib):
    assert binding.sa_linear_kernel_name(1, 0, 1, "none", 1, 0) == "unsupported"
    assert binding.sa_linear_kernel_name(100, 64, 64, "swiglu", 1, 0) != "unsupported"


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(3, 8), torch.zeros(4, 8)
    for call in (lambda: binding.sa_layer_norm_fwd(x), lambda: binding.sa_linear_fwd(x, w),
                 lambda: binding.sa_layer_norm_bwd(x, x, torch.zeros(3, 2)), lambda: binding.sa_linear_bwd(x, x, w)):
        with pytest.raises(ValueError, match="CUDA"):
            call()


def test_unknown_activation():
    with pytest.raises(ValueError, match="tanh"):
        binding._act("tanh")
