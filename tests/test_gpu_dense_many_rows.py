"""Norms and linear gradients over many rows: several rows for every block and every slot of its ring, column sums within a
bound that one row left out exceeds (tests/test_dense_bounds.py)."""
import pytest
import torch

import dense_sums as ds
from dense_cases import TORCH

pytestmark = pytest.mark.gpu

EPS = 1e-5

# at least six rows for a block's thread, twice the ring; nothing aligned, then aligned
SHAPES = [(120000, 63), (40000, 129), (30000, 333), (10007, 1001), (5000, 2047), (3000, 4097), (3000, 8191), (2000, 9001), (1500, 16383),
          (80013, 64), (80013, 128), (40000, 256), (20000, 512), (10007, 1024), (5000, 2048), (3000, 4096), (3000, 8192), (2000, 12000),
          (1500, 16384)]
TYPES = [("bf16", None, "bf16"), ("f32", "bf16", "f32"), ("bf16", "bf16", "f32"), ("f32", "f32", "f32"), ("f32", None, "bf16")]


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def inputs(rows, n, seed, x, r, y, stride=None):
    """x, r and dy as rows `stride` elements apart (contiguous by default), not on 16 bytes then."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*s):
        return torch.randn(s, generator=g, device="cuda")

    def matrix(dt, scale=False, offset=0.0):
        v = normal(rows, n)
        if scale:
            v = v * torch.exp(0.5 * normal(rows, 1)) + offset
        v = v.to(TORCH[dt])
        if stride is None:
            return v
        wide = torch.full((rows, stride), float("nan"), dtype=TORCH[dt], device="cuda")
        wide[:, 1:1 + n] = v
        return wide[:, 1:1 + n]

    return matrix(x, True, 0.5), None if r is None else matrix(r), (1 + 0.2 * normal(n)).to(TORCH[y]), \
        (0.2 * normal(n)).to(TORCH[y]), matrix(y)


def check_norm(b, x, r, w, bias, dy):
    y, stats = b.sa_layer_norm_fwd(x, w, bias, r, EPS, w.dtype, want_stats=True)
    dx, dr, dw, db = b.sa_layer_norm_bwd(dy, x, stats, w, r)
    ref = ds.norm_reference(*(None if v is None else v.double() for v in (x, r, w, bias, dy)), EPS, sms())
    for name, got, of in (("y", y, "y"), ("mean", stats[:, 0], "mean"), ("rstd", stats[:, 1], "rstd"), ("dx", dx, "dh"),
                          ("dr", dr, "dh"), ("dw", dw, "dw"), ("db", db, "db")):
        if got is not None:
            ds.check(name, got, *ref[of])


@pytest.mark.parametrize("types", TYPES, ids=str)
@pytest.mark.parametrize("rows,n", SHAPES)
def test_norm(cuda_lib, rows, n, types):
    check_norm(cuda_lib, *inputs(rows, n, rows + n, *types))


@pytest.mark.parametrize("rows,n,stride", [(40000, 128, 131), (10007, 1001, 1010), (5000, 2048, 2051), (3000, 8192, 8195)])
def test_norm_of_rows_apart(cuda_lib, rows, n, stride):
    """The shift of a row from 16 bytes is another for each row; nothing between the rows is taken."""
    for types in TYPES[:2]:
        check_norm(cuda_lib, *inputs(rows, n, n, *types, stride=stride))


@pytest.mark.parametrize("rows,n", [(10007, 1001), (120000, 63), (3000, 8191), (2000, 9001), (5000, 2048)])
def test_norm_in_place(cuda_lib, rows, n):
    b = cuda_lib
    x, r, w, bias, dy = inputs(rows, n, 3, "f32", "f32", "f32")
    ref = ds.norm_reference(*(v.double() for v in (x, r, w, bias, dy)), EPS, sms())
    stream = torch.cuda.current_stream().cuda_stream
    for into in (x.clone(), r.clone()):
        a, c = (into, r) if torch.equal(into, x) else (x, into)
        assert b.load().sa_layer_norm_fwd(a.data_ptr(), n, 0, c.data_ptr(), n, 0, w.data_ptr(), bias.data_ptr(), 0, rows, n, EPS,
                                          into.data_ptr(), 0, None, stream) == 0
        ds.check("y", into, *ref["y"])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "swiglu"])
@pytest.mark.parametrize("M,K,N", [(20011, 128, 128), (20011, 72, 131), (9001, 40, 600)])
def test_linear_gradients(cuda_lib, M, K, N, act, dt):
    b, t = cuda_lib, TORCH[dt]
    g = torch.Generator(device="cuda").manual_seed(M + N)
    Z = 2 * N if act == "swiglu" else N
    dy, x, w, z = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((M, N), (M, K), (Z, K), (M, Z)))
    dx, dw, db = b.sa_linear_bwd(dy, x, w, None if act == "none" else z, act)
    assert b.sa_linear_get_device_error() == 0
    dx64, dw64, (db64, e) = ds.linear_grad_reference(*(v.double() for v in (dy, x, w, z)), act, dt, sms())
    assert ds.spread(dx, dx64) <= 1.5 * ds.SPREAD[dt] and ds.spread(dw, dw64) <= 1.5 * ds.SPREAD[dt]
    ds.check("db", db, db64, e)
