"""Shared by the tests of layer norm and linear layers: inputs, and how far a kernel may be off, derived
from its roundings.

u = 2^-24 is half a step of fp32 and H(dt) half a step of the output's type (bf16 2^-8 / 2 = 2^-9... written
as eps / 2).  Sums of n terms in fp32, in any order and with truncating or rounding adders, are off by at most
2 n u times the sum of the terms' sizes."""
from __future__ import annotations

import numpy as np
import torch

from oracle import dense_oracle as do

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
U = 2.0 ** -24


def half_step(dt):
    return torch.finfo(TORCH[dt]).eps / 2


def rounded(x, dt):
    """x as the type holds it, in fp64."""
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TORCH[dt]).double().numpy()


def to_gpu(x, dt):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to("cuda", torch.float32).to(TORCH[dt])


def check(name, got, ref, most):
    got = got.detach().double().cpu().numpy() if torch.is_tensor(got) else np.asarray(got)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    assert np.all(np.isfinite(got)), f"{name}: not finite"
    over = np.abs(got - ref) - (most + 1e-30)
    assert not np.any(over > 0), (f"{name}: {int(np.sum(over > 0))} of {over.size} off by more than allowed, worst by "
                                  f"{over.max():.3e} at {np.unravel_index(over.argmax(), over.shape)}")


# ------------------------------------------------------------- layer norm

def norm_inputs(rows, n, seed, x="bf16", r=None, y="bf16", offset=0.5):
    rng = np.random.default_rng(seed)
    c = {"x": rounded(rng.standard_normal((rows, n)) * np.exp(0.5 * rng.standard_normal((rows, 1))) + offset, x),
         "r": None if r is None else rounded(rng.standard_normal((rows, n)), r),
         "w": rounded(1 + 0.2 * rng.standard_normal(n), y), "b": rounded(0.2 * rng.standard_normal(n), y),
         "dy": rounded(rng.standard_normal((rows, n)), y)}
    c["h"] = c["x"] if r is None else c["x"] + c["r"]
    return c


def norm_limits(c, eps, y="bf16"):
    """Bounds of y, mean and rstd.

    h is one sum of two fp32 numbers (u).  A thread adds at most 16 elements and the rows' threads join in at most ten
    steps, so the mean is off by 2 * 27 u of the mean size of h.  The differences from it inherit that and u of their
    own; their mean square is off by 2 * 27 u + 4 u relative from its sum and by the square of the mean's
    error (second order: taken as the differences' errors once more); 1/sqrt halves that and adds 2^-22 of its own."""
    h, n = c["h"], c["h"].shape[1]
    y64, mean, rstd = do.layer_norm(h, c["w"], c["b"], eps)
    size = np.abs(h).mean(1)
    e_mean = 56 * U * size + U * np.abs(mean)
    e_d = (U * np.abs(h) + e_mean[:, None]) * 1.01 + U * np.abs(h - mean[:, None])
    d2 = np.abs(h - mean[:, None])
    e_var = 60 * U * (d2 ** 2).mean(1) + 2 * (d2 * e_d).mean(1) + (e_d ** 2).mean(1)
    e_r = rstd * (0.5 * e_var * rstd ** 2 * 1.01 + 4 * U + 2.0 ** -22)
    xh = np.abs(h - mean[:, None]) * rstd[:, None]
    e_y = (e_d * rstd[:, None] + d2 * e_r[:, None] + 2 * U * xh) * np.abs(c["w"]) + U * np.abs(y64)
    return (y64, e_y * 1.01 + half_step(y) * (np.abs(y64) + e_y)), (mean, e_mean + U * size), (rstd, e_r)


def norm_grad_limits(c, eps, x="bf16", r=None, y="bf16", row_depth=None):
    """Bounds of dh (before its rounding to a type), dw and db.  The statistics are the forward's in fp32 (the
    errors above); sums over rows in fp32 are off by 2 * rows * u of their sizes."""
    h, w, dy = c["h"], c["w"], c["dy"]
    rows, n = h.shape
    dh, dw, db = do.layer_norm_grad(dy, h, w, eps)
    _, (mean, e_mean), (rstd, e_r) = norm_limits(c, eps, y)
    d2 = np.abs(h - mean[:, None])
    xh = d2 * rstd[:, None]
    e_xh = (U * np.abs(h) + e_mean[:, None] + U * d2) * rstd[:, None] + d2 * e_r[:, None] + U * xh
    g = np.abs(dy * w)
    e_g = U * g
    e_mg = 56 * U * g.mean(1) + e_g.mean(1)
    gx = g * xh
    e_mx = 60 * U * gx.mean(1) + (g * e_xh).mean(1)
    mg, mx = np.abs((dy * w).mean(1)), np.abs((dy * w * (h - mean[:, None]) * rstd[:, None]).mean(1))
    inner = g + mg[:, None] + xh * mx[:, None]
    e_dh = rstd[:, None] * (e_g + e_mg[:, None] + xh * e_mx[:, None] + e_xh * mx[:, None] + 4 * U * inner) + \
        e_r[:, None] * inner
    depth = 2 * (rows + 8) * U
    e_dw = (np.abs(dy) * e_xh).sum(0) + depth * (np.abs(dy) * xh).sum(0)
    e_db = depth * np.abs(dy).sum(0)
    hy = half_step(y)
    return (dh, 1.01 * e_dh), (dw, e_dw + hy * (np.abs(dw) + e_dw)), (db, e_db + hy * (np.abs(db) + e_db))


# ----------------------------------------------------------------- linear

def linear_inputs(M, K, N, act, dt, seed, bias=True, res=False, scale=1.0):
    rng = np.random.default_rng(seed)
    Z = 2 * N if act == "swiglu" else N
    c = {"x": rounded(rng.standard_normal((M, K)) * scale, dt),
         "w": rounded(rng.standard_normal((Z, K)) / np.sqrt(K), dt),
         "b": rounded(0.3 * rng.standard_normal(Z), dt) if bias else None,
         "r": rounded(rng.standard_normal((M, N)), dt) if res else None,
         "dy": rounded(rng.standard_normal((M, N)), dt)}
    return c


# Error of an activation and of its slope relative to 1 + |z|: bf16 results take the hardware's 2^x and 1/x and a
# polynomial that is off by 7.5e-6; fp32 results CUDA's functions (2 to 4 steps of fp32, some after a cancellation).
ACT_ERROR = {"bf16": 1.2e-5, "f32": 8 * U}


def linear_limits(c, act, dt):
    """Bounds of y and z.  Products of bf16 are exact in fp32; fp32 products of three bf16 terms each lose at most
    2^-22 of their size.  Slopes are at most 1.13, and |act(z)| at most |z|."""
    y, z = do.linear(c["x"], c["w"], c["b"], c["r"], act)
    size = np.abs(c["x"]) @ np.abs(c["w"]).T + (0 if c["b"] is None else np.abs(c["b"]))
    K = c["x"].shape[1]
    e_z = (2 * (K + 2) * U + (0 if dt == "bf16" else 2.0 ** -22)) * size
    if act == "swiglu":
        n = z.shape[1] // 2
        a, u = z[:, :n], z[:, n:]
        e_gate = 1.13 * e_z[:, :n] + ACT_ERROR[dt] * np.abs(do.activate(a, "silu")) + ACT_ERROR[dt] * e_z[:, :n]
        e_a = e_gate * (np.abs(u) + e_z[:, n:]) + np.abs(do.activate(a, "silu")) * (e_z[:, n:] + 2 * U * np.abs(u))
    elif act == "none":
        e_a = e_z
    else:
        e_a = 1.13 * e_z + ACT_ERROR[dt] * np.abs(do.activate(z, act))
        if act == "gelu":  # Phi comes out of 1 - R: off by ACT_ERROR of 1, times z
            e_a = 1.13 * e_z + ACT_ERROR[dt] * np.abs(z)
    h = half_step(dt)
    e_y = e_a + 2 * U * np.abs(y)
    return (y, e_y + h * (np.abs(y) + e_y)), (z, e_z + h * (np.abs(z) + e_z))


def linear_grad_limits(c, z, act, dt):
    """Bounds of dx, dw, db for the forward's z as the type holds it."""
    dx, dw, db, dz = do.linear_grad(c["dy"], c["x"], c["w"], z, act)
    M, K = c["x"].shape
    Z = c["w"].shape[0]
    h = half_step(dt)
    if act == "none":
        e_s = np.zeros_like(dz)
    elif act == "swiglu":
        n = z.shape[1] // 2
        a, u = z[:, :n], z[:, n:]
        g = np.abs(c["dy"])
        e_s = np.concatenate([g * np.abs(u) * ACT_ERROR[dt] * (1 + np.abs(a)), g * ACT_ERROR[dt] * np.abs(a)], 1)
    elif act == "relu":
        e_s = np.zeros_like(dz)
    else:
        e_s = np.abs(c["dy"]) * ACT_ERROR[dt] * (1 + np.abs(z))
    e_s = e_s + 4 * U * np.abs(dz)
    e_o = e_s + (0 if act in ("none", "relu") else h * (np.abs(dz) + e_s))  # as an operand, rounded to dt
    split = 0 if dt == "bf16" else 2.0 ** -22
    w, x = np.abs(c["w"]), np.abs(c["x"])
    s_dx, s_dw = np.abs(dz) @ w, np.abs(dz).T @ x
    e_dx = e_o @ w + (2 * (Z + 2) * U + split) * s_dx
    e_dw = e_o.T @ x + (2 * (M + 2) * U + split) * s_dw
    e_db = e_s.sum(0) + 2 * (M + 2) * U * np.abs(dz).sum(0)
    return tuple((v, e + h * (np.abs(v) + e)) for v, e in ((dx, e_dx), (dw, e_dw), (db, e_db)))
