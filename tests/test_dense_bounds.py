"""The bounds of tests/dense_sums.py see a single row that is left out of a column sum, and let fp32 sums in the kernels'
order pass (no GPU)."""
import numpy as np
import pytest
import torch

import dense_sums as ds

SMS = 152


def norm_case(rows, n, seed=0):
    g = torch.Generator().manual_seed(seed)
    def normal(*s):
        return torch.randn(s, generator=g).double()
    return normal(rows, n) * torch.exp(0.5 * normal(rows, 1)) + 0.5, normal(rows, n), 1 + 0.2 * normal(n), 0.2 * normal(n), normal(rows, n)


def summed(terms, at_once):
    """Column sums in fp32: threads over their rows, then blocks' rows one after the other."""
    blocks = SMS
    t = torch.zeros((-(-terms.shape[0] // (blocks * at_once)) * blocks * at_once, terms.shape[1]))
    t[:terms.shape[0]] = terms.float()
    t = t.view(-1, blocks * at_once, terms.shape[1])
    s = t[0].clone()
    for part in t[1:]:
        s += part
    out = torch.zeros(terms.shape[1])
    for part in s.view(-1, 32, terms.shape[1]) if s.shape[0] % 32 == 0 else s[:, None]:
        out += part.sum(0)
    return out


@pytest.mark.parametrize("rows,n", [(120000, 63), (80013, 128), (10007, 1001), (5000, 2047)])
def test_a_row_left_out_is_seen(rows, n):
    x, r, w, b, dy = norm_case(rows, n)
    ref = ds.norm_reference(x, r, w, b, dy, 1e-5, SMS)
    h = x + r
    xh = ((h - h.mean(1, keepdim=True)) * (h.var(1, keepdim=True, correction=0) + 1e-5).rsqrt()).float().double()
    at_once = next((k for most, k in ds.ROWS_AT_ONCE if n <= most), 1)
    for name, terms in (("dw", dy * xh), ("db", dy)):
        ds.check(name, summed(terms, at_once), *ref[name])
        for row in (0, rows // 2, rows - 1):
            short = terms.clone()
            short[row] = 0
            with pytest.raises(AssertionError, match=name):
                ds.check(name, summed(short, at_once), *ref[name])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu", "swiglu"])
def test_a_row_left_out_of_a_linear_gradient_is_seen(act, dt):
    M, K, N = 20011, 40, 24
    g = torch.Generator().manual_seed(1)
    t = {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
    Z = 2 * N if act == "swiglu" else N
    dy, x, z, w = (torch.randn(s, generator=g).to(t).double() for s in ((M, N), (M, K), (M, Z), (Z, K)))
    _, dw, (db, e) = ds.linear_grad_reference(dy, x, w, z, act, dt, SMS)
    assert ds.spread(dw.to(t), dw) <= ds.SPREAD[dt]
    ds.check("db", db.to(t), db, e)
    for row in dy.abs().sum(1).argsort()[M // 3:M:M // 5]:
        short = dy.clone()
        short[row] = 0
        _, dw1, (db1, _) = ds.linear_grad_reference(short, x, w, z, act, dt, SMS)
        assert ds.spread(dw1.to(t), dw) > 1.5 * ds.SPREAD[dt]
        with pytest.raises(AssertionError, match="db"):
            ds.check("db", db1.to(t), db, e)


def test_the_reference_is_the_oracle_s():
    from oracle import dense_oracle as do

    x, r, w, b, dy = norm_case(7, 33)
    ref = ds.norm_reference(x, r, w, b, dy, 1e-5, SMS)
    y, mean, rstd = do.layer_norm((x + r).numpy(), w.numpy(), b.numpy(), 1e-5)
    dh, dw, db = do.layer_norm_grad(dy.numpy(), (x + r).numpy(), w.numpy(), 1e-5)
    for name, v in (("y", y), ("mean", mean), ("rstd", rstd), ("dh", dh), ("dw", dw), ("db", db)):
        assert np.allclose(ref[name][0].numpy(), v, rtol=1e-12, atol=1e-12), name
    for act in do.ACTIVATIONS:
        Z = 12 if act == "swiglu" else 6
        g = torch.Generator().manual_seed(2)
        x, w, b, r, dy = (torch.randn(s, generator=g).double() for s in ((5, 4), (Z, 4), (Z,), (5, 6), (5, 6)))
        (y, _), (z, _) = ds.linear_reference(x, w, b, r, act, "f32")
        y64, z64 = do.linear(*(v.numpy() for v in (x, w, b, r)), act)
        assert np.allclose(y.numpy(), y64) and np.allclose(z.numpy(), z64)
        dx, dw, (db, _) = ds.linear_grad_reference(dy, x, w, z, act, "f32", SMS)
        for p, q in zip((dx, dw, db), do.linear_grad(*(v.numpy() for v in (dy, x, w, z)), act)):
            assert np.allclose(p.numpy(), q)
