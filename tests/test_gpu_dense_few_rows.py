"""bf16 gradients of few rows on either side of the choice between W read where it is and its aligned copy."""
import pytest
import torch

import dense_sums as ds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["none", "gelu", "swiglu"])
@pytest.mark.parametrize("M", [1, 3, 4, 5, 8, 15, 16])
@pytest.mark.parametrize("K", [333, 1024])
def test_gradients(cuda_lib, M, K, act):
    b, N = cuda_lib, 600
    g = torch.Generator(device="cuda").manual_seed(M + K)
    Z = 2 * N if act == "swiglu" else N
    wide = torch.randn((Z, K + 40), generator=g, device="cuda").mul_(K ** -0.5).bfloat16()
    dy, x, z = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((M, N), (M, K), (M, Z)))
    for w in (wide[:, :K].contiguous(), wide[:, 3:3 + K], wide[:, 8:8 + K]):
        dx, dw, db = b.sa_linear_bwd(dy, x, w, None if act == "none" else z, act)
        assert b.sa_linear_get_device_error() == 0
        dx64, dw64, (db64, e) = ds.linear_grad_reference(*(v.double() for v in (dy, x, w, z)), act, "bf16",
                                                         torch.cuda.get_device_properties(0).multi_processor_count)
        assert ds.spread(dx, dx64) <= 1.5 * ds.SPREAD["bf16"] and ds.spread(dw, dw64) <= 1.5 * ds.SPREAD["bf16"]
        ds.check("db", db, db64, e)
