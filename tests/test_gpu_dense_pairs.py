"""Linear layers on pairs of CTAs: every end of a tile, whole and cut, with and without z and residual, rows that 16-byte
pieces fit and rows that they do not.  Which kernels ran is asserted, by name and by the number of launches."""
import pytest
import torch

import dense_sums as ds

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "silu", "swiglu"]


def case(M, K, N, act, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + M + N)
    Z = 2 * N if act == "swiglu" else N
    return tuple(torch.randn(s, generator=g, device="cuda").mul_(f).bfloat16() for s, f in (
        ((M, K), 1), ((Z, K), K ** -0.5), ((Z,), 0.3), ((M, N), 1), ((M, N), 1)))


def check(b, x, w, bias, r, act, kind, launches, pre=True):
    M, K = x.shape
    N = w.shape[0] // (2 if act == "swiglu" else 1)
    assert b.sa_linear_kernel_name(M, N, K, act, b.SA_BF16, 0) == kind
    before = b.sa_launch_count()
    got = b.sa_linear_fwd(x, w, bias, act, r, want_pre=pre)
    assert b.sa_launch_count() - before == launches
    assert b.sa_linear_get_device_error() == 0
    (y64, e_y), (z64, e_z) = ds.linear_reference(*(None if v is None else v.double() for v in (x, w, bias, r)), act, "bf16")
    y, z = got if pre else (got, None)
    for name, v, ref, e in (("y", y, y64, e_y), ("z", z, z64, e_z)):
        if v is not None:
            ds.check(name, v, ref, e)
            assert ds.spread(v, ref) <= ds.SPREAD["bf16"]
    return z


# whole tiles, or cut ones too (1: a join); aligned rows and others
SHAPES = [(2048, 1024, 2048, 0), (2304, 4096, 2304, 1), (2400, 2048, 2104, 0), (2400, 2048, 2100, 1), (1280, 8192, 1280, 1)]
GATED = [(2048, 1024, 2048, 0), (700, 8192, 520, 1), (700, 8192, 519, 1), (2048, 1024, 2052, 0), (2400, 2048, 2100, 1)]


@pytest.mark.parametrize("act,shape", [(a, s) for a in ACTS for s in (GATED if a == "swiglu" else SHAPES)], ids=str)
def test_ends(cuda_lib, act, shape):
    M, K, N, joins = shape
    x, w, bias, r, _ = case(M, K, N, act)
    for b_, r_, pre in ((bias, r, True), (None, None, False), (bias, None, True), (None, r, False)):
        check(cuda_lib, x, w, b_, r_, act, "tc5_linear_pair", 1 + joins, pre)


@pytest.mark.parametrize("act", ACTS)
def test_a_residual_that_no_16_byte_pieces_fit(cuda_lib, act):
    """y's rows leave by TMA, the residual comes element by element."""
    x, w, bias, r, _ = case(2048, 1024, 2048, act)
    wide = torch.zeros((2048, 2051), dtype=torch.bfloat16, device="cuda")
    wide[:, 3:] = r
    check(cuda_lib, x, w, bias, wide[:, 3:], act, "tc5_linear_pair", 1)


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("M,K,N", [(4096, 1024, 4096), (4096, 1023, 4096), (2400, 2048, 2104),
                                   (5000, 1024, 2600)])
def test_gradients(cuda_lib, M, K, N, act):
    b = cuda_lib
    x, w, bias, _, dy = case(M, K, N, act)
    assert all(b.sa_linear_kernel_name(M, N, K, act, b.SA_BF16, i) == "tc5_linear_pair" for i in (1, 2))
    _, z = b.sa_linear_fwd(x, w, bias, act, want_pre=True)
    z = x @ w.T if z is None else z
    dx64, dw64, (db64, e) = ds.linear_grad_reference(*(v.double() for v in (dy, x, w, z)), act, "bf16",
                                                     torch.cuda.get_device_properties(0).multi_processor_count)
    whole = b.sa_linear_bwd(dy, x, w, z, act)
    alone = b.sa_linear_bwd(dy, x, w, z, act, True, False, False)[0], b.sa_linear_bwd(dy, x, w, z, act, False, True, False)[1]
    assert b.sa_linear_get_device_error() == 0
    for dx, dw in (whole[:2], alone):
        assert ds.spread(dx, dx64) <= 1.5 * ds.SPREAD["bf16"] and ds.spread(dw, dw64) <= 1.5 * ds.SPREAD["bf16"]
    ds.check("db", whole[2], db64, e)
