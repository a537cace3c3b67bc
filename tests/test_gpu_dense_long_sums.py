"""Long sums of one sign in bf16 layers.

The tensor core's additions (of 16 products each) lose up to two steps of fp32, 2^-23 relative, always towards zero, of a sum
that is on average half as large as it ends. At most 1024 of them go into an accumulator before it is added to sums that
round to nearest, so results are less than 1024 * 2 * 2^-23 / 2 = 2^-13 too small on average, however many terms they
have. The results' own roundings spread evenly over their steps, since rows and columns are scaled differently: up to 2^-8
relative either way, 2^-8 / sqrt(3) a result, and over n results their mean stays within four times 2^-8 / sqrt(3 n)."""
import pytest
import torch

pytestmark = pytest.mark.gpu

def limit(results):
    return 2.0 ** -13 + 4 * 2.0 ** -8 / (3 * results) ** 0.5


def positive(rows, cols, seed, scale_rows):
    """Sizes of a normal distribution; scaled by 1 to 4 along the axis that stays."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    v = torch.rand((rows, 1) if scale_rows else (1, cols), generator=g, device="cuda")
    out = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for i in range(0, rows, 4096):
        n = min(4096, rows - i)
        part = torch.randn((n, cols), generator=g, device="cuda").abs_()
        out[i:i + n] = part.mul_(torch.exp2(2 * (v[i:i + n] if scale_rows else v)))
    return out


def exact(a, b):
    """a^T b in 64 bits, a [k, m], b [k, n]"""
    ref = torch.zeros((a.shape[1], b.shape[1]), dtype=torch.float64, device="cuda")
    for i in range(0, a.shape[0], 16384):
        ref += a[i:i + 16384].double().T @ b[i:i + 16384].double()
    return ref


def off(got, ref):
    """Mean relative difference"""
    return float(((got.double() - ref) / ref).mean())


@pytest.mark.parametrize("M,K,N,kind", [(200003, 2048, 2048, "tc5_linear_pair"), (200003, 1000, 1200, "tc5_linear_pair"),
                                        (12000011, 128, 128, "tc5_linear")])
def test_weight_gradient_over_many_rows(cuda_lib, M, K, N, kind):
    b = cuda_lib
    dy, x = positive(M, N, 1, False), positive(M, K, 2, False)
    w = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda")
    assert b.sa_linear_kernel_name(M, N, K, "none", 1, 2) == kind
    alone = b.sa_linear_bwd(dy, x, w, want_dx=False, want_db=False)[1]
    dw, db = b.sa_linear_bwd(dy, x, w)[1:]
    assert b.sa_linear_get_device_error() == 0
    ref = exact(dy, x)
    for got in (alone, dw):
        assert abs(off(got, ref)) <= limit(K * N), off(got, ref)
    ref = sum(dy[i:i + 65536].double().sum(0) for i in range(0, M, 65536))
    assert float((db.double() / ref - 1).abs().max()) <= 2.0 ** -8 + 1e-5


@pytest.mark.parametrize("M,K,N,kind", [(2048, 200008, 2048, "tc5_linear_pair"), (640, 1000003, 640, "tc5_linear_pair")])
def test_forward_over_many_features(cuda_lib, M, K, N, kind):
    b = cuda_lib
    x, w = positive(M, K, 3, True), positive(N, K, 4, True)
    assert b.sa_linear_kernel_name(M, N, K, "none", 1, 0) == kind
    y = b.sa_linear_fwd(x, w)
    assert b.sa_linear_get_device_error() == 0
    ref = exact(x.T, w.T)
    assert abs(off(y, ref)) <= limit(M * N), off(y, ref)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu", "swiglu"])
def test_activations_behind_long_sums(cuda_lib, act):
    """The end of a tile after several runs: bias, activation, residual and z, one CTA and pairs."""
    b, K = cuda_lib, 40960
    for M, N in ((2304, 2048), (700, 520)):
        g = torch.Generator(device="cuda").manual_seed(N)
        Z = 2 * N if act == "swiglu" else N
        x = torch.randn((M, K), generator=g, device="cuda").bfloat16()
        w = torch.randn((Z, K), generator=g, device="cuda").mul_(K ** -0.5).bfloat16()
        bias, r = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((Z,), (M, N)))
        y, z = b.sa_linear_fwd(x, w, bias, act, r, want_pre=True)
        assert b.sa_linear_get_device_error() == 0
        z64 = x.double() @ w.double().T + bias.double()
        f = torch.nn.functional
        y64 = {"relu": f.relu, "gelu": f.gelu, "silu": f.silu,
               "swiglu": lambda v: f.silu(v[:, :N]) * v[:, N:]}[act](z64) + r.double()
        for got, ref in ((z, z64), (y, y64)):  # roundings spread evenly over their steps, 2^-9 / sqrt(3)
            assert float((got.double() - ref).norm() / ref.norm()) <= 2.0 ** -9


@pytest.mark.parametrize("M", [1, 16])
def test_few_rows_of_many_features(cuda_lib, M):
    b, K, N = cuda_lib, 1 << 20, 4096
    x, w = positive(M, K, 5, True), positive(N, K, 6, True)
    assert b.sa_linear_kernel_name(M, N, K, "none", 1, 0) == "mma_linear_rows"
    y = b.sa_linear_fwd(x, w)
    ref = exact(x.T, w.T)
    assert abs(off(y, ref)) <= limit(M * N), off(y, ref)


def test_input_gradient_over_many_columns(cuda_lib):
    b, M, K, N = cuda_lib, 2048, 2048, 200008
    dy, w = positive(M, N, 7, True), positive(N, K, 8, False)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    dx = b.sa_linear_bwd(dy, x, w, want_dw=False, want_db=False)[0]
    assert b.sa_linear_get_device_error() == 0
    ref = exact(dy.T, w)
    assert abs(off(dx, ref)) <= limit(M * K), off(dx, ref)
