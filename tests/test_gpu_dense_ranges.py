"""fp32 linear layers at the ends of the type's range.

On the tensor cores a factor is three bf16 terms. Their sum is the factor for sizes from 2^-110 up to the largest finite one;
below 2^-110 what lies under half of bf16's smallest subnormal, 2^-134, is lost, and nothing else."""
import numpy as np
import pytest
import torch

import dense_cases as dc

pytestmark = pytest.mark.gpu

MOST = float(np.finfo(np.float32).max)
# the largest values; the smallest that rounds to no finite bf16, and its neighbour below; bf16's largest
LARGE = [MOST, -MOST, 3.3961775e38, 3.3961773e38, 3.3895314e38, -3.39e38]


def put(a, values):
    """One of the values in every third row, in columns of its own."""
    for i in range(0, a.shape[0], 3):
        a[i, (5 * i + 1) % a.shape[1]] = np.float32(values[i % len(values)])


@pytest.mark.parametrize("M", [16, 17, 200])
@pytest.mark.parametrize("K,N", [(128, 96), (101, 97)])
@pytest.mark.parametrize("act", ["none", "relu", "silu"])
def test_the_largest_values(cuda_lib, M, K, N, act):
    """y for such x, and for such W; dx and dW for such dy, by way of copies and of the activation's slope."""
    b = cuda_lib
    c = dc.linear_inputs(M, K, N, act, "f32", M + K)
    c["w"] = dc.rounded(c["w"] * 1e-3, "f32")
    c["b"] = dc.rounded(np.full(N, 100.0), "f32")  # z is positive where no large value is
    put(c["x"], LARGE)
    t = {k: dc.to_gpu(v, "f32") for k, v in c.items()}
    y = b.sa_linear_fwd(t["x"], t["w"], t["b"], act)
    (y64, e), _ = dc.linear_limits(c, act, "f32")
    dc.check("y", y, y64, e)

    swapped = dict(c, x=c["w"], w=c["x"], b=None, r=None)
    y = b.sa_linear_fwd(t["w"], t["x"])
    (y64, e), _ = dc.linear_limits(swapped, "none", "f32")
    dc.check("y of large W", y, y64, e)

    c = dc.linear_inputs(M, K, N, act, "f32", M + K + 1)
    c["x"], c["w"] = (dc.rounded(c[k] * 1e-3, "f32") for k in ("x", "w"))
    put(c["dy"], [v / 2 for v in LARGE] if act == "silu" else LARGE)
    z = dc.rounded(np.full((M, N), 60.0), "f32")  # slopes of 1
    t = {k: dc.to_gpu(v, "f32") for k, v in c.items()}
    got = b.sa_linear_bwd(t["dy"], t["x"], t["w"], dc.to_gpu(z, "f32"), act, want_db=False)
    assert b.sa_linear_get_device_error() == 0
    for name, v, (ref, e) in zip(("dx", "dw"), got, dc.linear_grad_limits(c, z, act, "f32")):
        dc.check(name, v, ref, e)


@pytest.mark.parametrize("M", [16, 17, 200])
@pytest.mark.parametrize("power", [-60, -100, -110, -118])
def test_small_values(cuda_lib, M, power):
    b = cuda_lib
    K, N = 128, 96
    c = dc.linear_inputs(M, K, N, "none", "f32", 9, bias=False)
    x = c["x"]
    for small in ("x", "w"):
        c["x"], c["w"] = (x * 2.0 ** power, dc.rounded(c["w"], "f32")) if small == "x" else (x, c["w"] * 2.0 ** power)
        c["x"], c["w"] = dc.rounded(c["x"], "f32"), dc.rounded(c["w"], "f32")
        y = b.sa_linear_fwd(dc.to_gpu(c["x"], "f32"), dc.to_gpu(c["w"], "f32"))
        (y64, e), _ = dc.linear_limits(c, "none", "f32")
        lost = 2.0 ** -134 * ((np.abs(c["w"]) > 0).sum(1)[None, :] * np.abs(c["x"]).max(1)[:, None] if small == "w"
                              else np.abs(c["w"]).sum(1)[None, :])
        over = np.abs(y.double().cpu().numpy() - y64) - (e + lost)
        assert over.max() <= 0, (small, over.max(), np.abs(y64).max())


@pytest.mark.parametrize("M", [17, 200])
def test_an_infinity_or_nan_is_seen(cuda_lib, M):
    """With more than 16 rows an infinite factor makes a NaN, never a finite result."""
    b = cuda_lib
    x, w = torch.randn((M, 128), device="cuda"), torch.randn((96, 128), device="cuda")
    x[3, 7], x[5, 9], w[11, 2] = float("inf"), float("nan"), float("-inf")
    y = b.sa_linear_fwd(x, w)
    bad = torch.zeros((M, 96), dtype=torch.bool, device="cuda")
    bad[3], bad[5], bad[:, 11] = True, True, True
    assert torch.equal(~torch.isfinite(y), bad)
    dy = torch.randn((M, 96), device="cuda")
    dy[3, 1] = float("inf")
    dx, dw, _ = b.sa_linear_bwd(dy, torch.randn_like(x), torch.randn_like(w))
    rows = torch.arange(M, device="cuda") == 3
    columns = torch.arange(96, device="cuda") == 1
    assert torch.equal(~torch.isfinite(dx), rows[:, None].expand(M, 128))
    assert torch.equal(~torch.isfinite(dw), columns[:, None].expand(96, 128))
