"""The stacked refinement's layers run together, against the same formulas in 64 bits, with all gradients."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def reference(state, X, cu, layer, scale, eps=1e-5):
    """fp64, per user and head, by the formulas."""
    def norm(h, w, b):
        m = h.mean(-1, keepdim=True)
        return (h - m) / ((h - m).square().mean(-1, keepdim=True) + eps).sqrt() * w + b

    out = []
    for u in range(len(cu) - 1):
        x = X[cu[u]:cu[u + 1]]
        heads = []
        for h in range(X.shape[1]):
            q, k = state[u, h] @ layer.w_q.T, x[:, h] @ layer.w_k.T
            heads.append(torch.softmax(scale * q @ k.T, 0) @ x[:, h] if len(x) else torch.zeros_like(state[u, h]))
        out.append(torch.stack(heads))
    x1 = norm(state + torch.stack(out), layer.norm1_w, layer.norm1_b)
    a, g = (x1 @ layer.w_in.T).chunk(2, -1)
    return norm(x1 + (torch.nn.functional.silu(a) * g) @ layer.w_out.T, layer.norm2_w, layer.norm2_b)


@pytest.mark.parametrize("dtype,P,d,most", [(torch.bfloat16, 128, 64, 2e-2), (torch.bfloat16, 256, 128, 2e-2),
                                            (torch.float32, 48, 32, 1e-4)])
def test_two_layers_against_64_bits(cuda_lib, dtype, P, d, most):
    """Relative in the 2-norm: bf16 rounds every step's result (2^-9 each, some ten steps deep), fp32 1e-4 as the
    sketching step's own tolerance."""
    from paper_2609_08443_gb300 import refine

    gen = torch.Generator(device="cuda").manual_seed(P)
    lens, H = [300, 0, 77, 1], 2
    cu = torch.tensor([0, 300, 300, 377, 378], dtype=torch.int32, device="cuda")
    X = torch.randn((sum(lens), H, d), generator=gen, device="cuda").to(dtype).requires_grad_(True)
    state = torch.randn((len(lens), H, P, d), generator=gen, device="cuda").to(dtype).requires_grad_(True)
    layers = [refine.RefineLayer(*(w.requires_grad_(True) for w in refine.random_layer(d, 2 * d, dtype, generator=gen)))
              for _ in range(2)]
    dy = torch.randn(state.shape, generator=gen, device="cuda").to(dtype)
    out = refine.sa_refine(state, X, cu, layers)
    assert out.dtype is dtype and out.shape == state.shape
    out.backward(dy)

    X64, s64 = X.detach().double().requires_grad_(True), state.detach().double().requires_grad_(True)
    l64 = [refine.RefineLayer(*(w.detach().double().requires_grad_(True) for w in l)) for l in layers]
    ref = s64
    for l in l64:
        ref = reference(ref, X64, cu.tolist(), l, 1 / math.sqrt(d))
    ref.backward(dy.double())

    def off(a, b):
        a, b = a.detach().double(), b.detach()
        return float((a - b).norm() / b.norm())

    assert off(out, ref) < most
    for name, a, b in (("X", X, X64), ("state", state, s64)):
        assert off(a.grad, b.grad) < 3 * most, name
    for l, m in zip(layers, l64):
        for name, a, b in zip(l._fields, l, m):
            assert off(a.grad, b.grad) < 3 * most, name


def test_the_example_with_refinement(cuda_lib):
    from paper_2609_08443_gb300 import cached_targets

    plain = cached_targets.run(lengths=(900, 300, 130), H=2, P=128, d=64, candidates=70)
    again = cached_targets.run(lengths=(900, 300, 130), H=2, P=128, d=64, candidates=70, layers=2)
    assert torch.isfinite(again["z"]).all() and torch.isfinite(again["dq"]).all() and again["dq"].any()
    assert again["z"].shape == plain["z"].shape and not torch.equal(again["z"], plain["z"])
    assert torch.equal(again["recent"], plain["recent"])
