"""The fp64 reference of layer norm and linear layers against loops, differences and closed forms."""
import math

import numpy as np
import pytest

from oracle import dense_oracle as do

RNG = np.random.default_rng(3)


def differences(f, x, g, step=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        d = np.zeros_like(x)
        d[i] = step
        out[i] = (np.sum(g * f(x + d)) - np.sum(g * f(x - d))) / (2 * step)
    return out


def test_layer_norm_by_loops():
    h, w, b = RNG.standard_normal((3, 5)), RNG.standard_normal(5), RNG.standard_normal(5)
    y, mean, rstd = do.layer_norm(h, w, b, 0.01)
    for i in range(3):
        m = math.fsum(h[i]) / 5
        v = math.fsum((a - m) ** 2 for a in h[i]) / 5
        for j in range(5):
            assert y[i, j] == pytest.approx((h[i, j] - m) / math.sqrt(v + 0.01) * w[j] + b[j], rel=1e-13)
        assert mean[i] == pytest.approx(m) and rstd[i] == pytest.approx(1 / math.sqrt(v + 0.01))


def test_layer_norm_closed_forms():
    y, _, rstd = do.layer_norm(np.full((2, 7), 3.5), 2.0, np.arange(7.0), 1e-4)
    assert np.allclose(y, np.arange(7.0)) and np.allclose(rstd, 100)
    h = RNG.standard_normal((2, 6))
    assert np.allclose(do.layer_norm(h * 3 + 11, 1, 0, 0)[0], do.layer_norm(h, 1, 0, 0)[0])


def test_layer_norm_grad_by_differences():
    h, w, g = RNG.standard_normal((3, 6)), RNG.standard_normal(6), RNG.standard_normal((3, 6))
    dh, dw, db = do.layer_norm_grad(g, h, w, 1e-3)
    assert np.allclose(dh, differences(lambda a: do.layer_norm(a, w, 0, 1e-3)[0], h, g), atol=1e-7)
    assert np.allclose(dw, differences(lambda a: do.layer_norm(h, a, 0, 1e-3)[0], w, g), atol=1e-7)
    assert np.allclose(db, g.sum(0)) and np.allclose(dh.sum(1), 0, atol=1e-12)


@pytest.mark.parametrize("act", do.ACTIVATIONS)
def test_linear_by_differences(act):
    x, w, b, r = (RNG.standard_normal(s) for s in ((4, 3), (6, 3), (6,), (4, 3 if act == "swiglu" else 6)))
    g = RNG.standard_normal(r.shape)
    y, z = do.linear(x, w, b, r, act)
    dx, dw, db, _ = do.linear_grad(g, x, w, z, act)
    assert np.allclose(dx, differences(lambda a: do.linear(a, w, b, r, act)[0], x, g), atol=1e-7)
    assert np.allclose(dw, differences(lambda a: do.linear(x, a, b, r, act)[0], w, g), atol=1e-7)
    assert np.allclose(db, differences(lambda a: do.linear(x, w, a, r, act)[0], b, g), atol=1e-7)


def test_activations_at_points():
    z = np.array([[-3.0, -0.5, 0.0, 0.5, 3.0]])
    assert np.allclose(do.activate(z, "gelu"), [[v * 0.5 * (1 + math.erf(v / math.sqrt(2))) for v in z[0]]])
    assert np.allclose(do.activate(z, "silu"), [[v / (1 + math.exp(-v)) for v in z[0]]])
    two = np.array([[1.5, -2.0, 4.0, 0.25]])
    assert np.allclose(do.activate(two, "swiglu"),
                       [[1.5 / (1 + math.exp(-1.5)) * 4.0, -2 / (1 + math.exp(2)) * 0.25]])
