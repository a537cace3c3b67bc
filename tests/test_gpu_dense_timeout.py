"""A bounded wait of the linear layers' tensor-core kernels that runs out: failure detection without a GPU fault.

A limit below 1 ms makes the warp that issues the products wait for a barrier that nothing completes, so it gives up. The
worker's other roles then stop, the loads that were asked for land, the accumulators are freed, cut tiles are not joined, and
the call's workspace says SA_ERR_TIMEOUT. With the limit back, the next call in the same workspace gives the same bits as
before."""
import pytest
import torch

import dense_cases as dc

pytestmark = pytest.mark.gpu

SA_ERR_TIMEOUT = 5

# (M, K, N, activation, type), kernels of y, dx, dW: whole and cut tiles, one CTA, pairs, fp32, gradients side by side
# and one after the other
CASES = [((300, 136, 264, "swiglu", "bf16"), ("tc5_linear", "tc5_linear", "tc5_linear")),
         ((300, 4096, 520, "gelu", "bf16"), ("tc5_linear", "tc5_linear", "tc5_linear")),
         ((20000, 128, 512, "swiglu", "bf16"), ("tc5_linear", "tc5_linear", "tc5_linear")),
         ((2400, 2048, 2104, "gelu", "bf16"), ("tc5_linear_pair", "tc5_linear_pair", "tc5_linear_pair")),
         ((2400, 2048, 2100, "gelu", "bf16"), ("tc5_linear_pair", "tc5_linear_pair", "tc5_linear_pair")),
         ((4096, 1024, 4096, "none", "bf16"), ("tc5_linear_pair", "tc5_linear_pair", "tc5_linear_pair")),
         ((512, 128, 512, "gelu", "f32"), ("tc5_linear_f32",) * 3),
         ((1003, 509, 777, "swiglu", "f32"), ("tc5_linear_f32",) * 3)]


@pytest.mark.parametrize("case,kinds", CASES, ids=["-".join(map(str, c)) for c, _ in CASES])
def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean(cuda_lib, case, kinds):
    b = cuda_lib
    M, K, N, act, dt = case
    t = dc.TORCH[dt]
    assert tuple(b.sa_linear_kernel_name(M, N, K, act, b._dt_of(t), i) for i in range(3)) == kinds
    g = torch.Generator(device="cuda").manual_seed(M)
    Z = 2 * N if act == "swiglu" else N
    x, w, bias, r, dy = (torch.randn(s, generator=g, device="cuda").to(t) for s in ((M, K), (Z, K), (Z,), (M, N), (M, N)))
    size = max(b.load().sa_linear_workspace_size(M, N, K, b.SA_ACT[act], b._dt_of(t), i, 7) for i in (0, 1))
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def forward():
        return b.sa_linear_fwd(x, w, bias, act, r, want_pre=True, ws=ws)

    def backward():
        return b.sa_linear_bwd(dy, x, w, pre, act, ws=ws)

    y, pre = (None if v is None else v.clone() for v in forward())
    assert b.sa_get_device_error(ws) == 0
    grads = [v.clone() for v in backward()]
    assert b.sa_get_device_error(ws) == 0
    for call in (forward, backward):
        statuses = []
        try:
            b.sa_set_wait_limit_ns(1)
            for _ in range(3):
                call()
                statuses.append(b.sa_get_device_error(ws))
                if statuses[-1] == SA_ERR_TIMEOUT:
                    break
        finally:
            b.sa_set_wait_limit_ns(0)  # back to the default limit
        assert SA_ERR_TIMEOUT in statuses, statuses
        y2, pre2 = forward()
        assert b.sa_get_device_error(ws) == 0
        assert torch.equal(y, y2) and (pre is None or torch.equal(pre, pre2))
        again = backward()
        assert b.sa_get_device_error(ws) == 0
        assert all(torch.equal(p, q) for p, q in zip(grads, again))


def test_calls_without_waits_do_not_run_out(cuda_lib):
    """Few rows, products on CUDA cores and norms wait for nothing."""
    b = cuda_lib
    x, w = torch.randn((5, 64), device="cuda"), torch.randn((32, 64), device="cuda")
    try:
        b.sa_set_wait_limit_ns(1)
        b.sa_linear_bwd(b.sa_linear_fwd(x, w), x, w)
        assert b.sa_linear_get_device_error() == 0
        _, stats = b.sa_layer_norm_fwd(x, want_stats=True)
        b.sa_layer_norm_bwd(x, x, stats)
    finally:
        b.sa_set_wait_limit_ns(0)
    torch.cuda.synchronize()
