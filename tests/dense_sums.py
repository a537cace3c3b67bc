"""Bounds for long column sums and for large products, on whatever device the inputs are, in torch's fp64.

`dense_cases` bounds a column sum by twice the rows times u = 2^-24 of its terms' sizes, which at ten thousands of rows is more
than a row's term.  Here the bound is the depth of the additions, so that one row left out exceeds it."""
from __future__ import annotations

import torch

from dense_cases import ACT_ERROR, U

ROWS_AT_ONCE = ((64, 64), (128, 32), (256, 16), (512, 8))  # of a block, for up to so many features; else 1


def depth(rows, n, sms):
    """Additions that a term of a column sum goes through, at most: those of its thread (at least one block an SM), of the
    threads of a warp and the warps of a block that hold the same columns (3 + 8), and of the blocks' partial rows (every 32nd,
    of at most eight blocks an SM, then 32)."""
    at_once = next((r for most, r in ROWS_AT_ONCE if n <= most), 1)
    return -(-rows // (sms * at_once)) + 11 + -(-8 * sms // 32) + 32


def norm_reference(x, r, w, b, dy, eps, sms):
    """name -> (value, bound before the result's own rounding) for fp64 tensors x, r (or None), dy [rows, n], w, b [n].

    A thread adds at most 32 elements of a row and its threads join in at most ten steps: 2 * 43 u of the mean size of what is
    added, by the argument in dense_cases.  The sums of dw take terms whose errors e (of the row's own statistics) are independent of
    dy's signs: they add up in squares, and four times that is allowed; every addition rounds to nearest, u of a partial sum."""
    h = x if r is None else x + r
    mean = h.mean(1, keepdim=True)
    d = h - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    xh = d * rstd
    e_mean = 88 * U * h.abs().mean(1, keepdim=True) + U * mean.abs()
    e_d = 1.01 * (U * h.abs() + e_mean) + U * d.abs()
    e_var = 92 * U * var + 2 * (d.abs() * e_d).mean(1, keepdim=True) + (e_d * e_d).mean(1, keepdim=True)
    e_r = rstd * (0.505 * e_var * rstd ** 2 + 4 * U + 2.0 ** -22)
    e_xh = e_d * rstd + d.abs() * e_r + U * xh.abs()
    y = xh * w + b
    out = {"y": (y, 1.01 * ((e_xh + 2 * U * xh.abs()) * w.abs() + U * y.abs())),
           "mean": (mean[:, 0], (e_mean + U * h.abs().mean(1, keepdim=True))[:, 0]), "rstd": (rstd[:, 0], e_r[:, 0])}
    g = dy * w
    mg, mx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    gx = (g * xh).abs()
    e_mg = 89 * U * g.abs().mean(1, keepdim=True)
    e_mx = 92 * U * gx.mean(1, keepdim=True) + (g.abs() * e_xh).mean(1, keepdim=True)
    inner = g.abs() + mg.abs() + xh.abs() * mx.abs()
    out["dh"] = (rstd * (g - mg - xh * mx), 1.01 * (rstd * (U * g.abs() + e_mg + xh.abs() * e_mx + e_xh * mx.abs() + 4 * U * inner)
                                                 + e_r * inner))
    D = depth(*x.shape, sms) * U
    out["dw"] = ((dy * xh).sum(0), (D + 2 * U) * (dy * xh).abs().sum(0) + 4 * (dy * e_xh).square().sum(0).sqrt())
    out["db"] = (dy.sum(0), D * dy.abs().sum(0))
    return out


def check(name, got, ref, bound):
    assert got.shape == ref.shape and bool(torch.isfinite(got).all()), name
    half = torch.finfo(got.dtype).eps / 2
    over = (got.double() - ref).abs() - (bound + half * (ref.abs() + bound) + 1e-30)
    worst = float(over.max())
    assert worst <= 0, f"{name}: {int((over > 0).sum())} of {over.numel()} off by more than allowed, worst by {worst:.3e}"


def activate(z, act):
    f = torch.nn.functional
    if act == "swiglu":
        n = z.shape[1] // 2
        return f.silu(z[:, :n]) * z[:, n:]
    return {"none": lambda v: v, "relu": f.relu, "gelu": f.gelu, "silu": f.silu}[act](z)


def linear_reference(x, w, b, r, act, dt):
    """y and z with their bounds as in dense_cases.linear_limits, for fp64 tensors."""
    K = x.shape[1]
    z, size = x @ w.T, x.abs() @ w.abs().T
    if b is not None:
        z, size = z + b, size + b.abs()
    e_z = (2 * (K + 2) * U + (0 if dt == "bf16" else 2.0 ** -22)) * size
    a = activate(z, act)
    err = ACT_ERROR[dt]
    if act == "none":
        e = e_z
    elif act == "swiglu":
        n = z.shape[1] // 2
        s, u, e_s, e_u = activate(z[:, :n], "silu").abs(), z[:, n:].abs(), e_z[:, :n], e_z[:, n:]
        e = (1.13 * e_s + err * s + err * e_s) * (u + e_u) + s * (e_u + 2 * U * u)
    else:
        e = 1.13 * e_z + err * (z.abs() if act == "gelu" else a.abs())
    y = a if r is None else a + r
    return (y, e + 2 * U * y.abs()), (z, e_z)


def linear_grad_reference(dy, x, w, z, act, dt, sms):
    """(dx, dW) in fp64 by differentiation, and db with its bound: the sums' depth, and four times the squares' sum of the slopes'
    errors, which come with dy's signs (as in dense_cases.linear_grad_limits)."""
    z = z.detach().requires_grad_()
    dz, = torch.autograd.grad(activate(z, act), z, dy)
    z, err, g = z.detach(), ACT_ERROR[dt], dy.abs()
    if act in ("none", "relu"):
        e = torch.zeros_like(dz)
    elif act == "swiglu":
        n = z.shape[1] // 2
        a, u = z[:, :n].abs(), z[:, n:].abs()
        e = torch.cat([g * u * err * (1 + a), g * err * a], 1)
    else:
        e = g * err * (1 + z.abs())
    e = e + 4 * U * dz.abs()
    rows, n = dy.shape
    lanes = next((k for k in (1, 2, 4, 8, 16) if 8 * k >= n), 32)
    strips = -(-n // 256)
    blocks = -(-8 * sms // strips)
    D = -(-rows // (8 * (32 // lanes) * blocks)) + 5 + 8 + -(-blocks // 32) + 32
    return dz @ w, dz.T @ x, (dz.sum(0), D * U * dz.abs().sum(0) + 4 * e.square().sum(0).sqrt())


def spread(got, ref):
    """Difference relative to the reference, norm-wise."""
    return float((got.double() - ref).norm() / ref.norm())


# Roundings to bf16 spread evenly over half steps of 2^-9 to 2^-8: over many results at most 2^-8 / sqrt(3) norm-wise if all had the
# largest step, 1.7e-3 as they come, 2^-9 with room for the sums; half as much again where dz was rounded as an operand.
# Sums of fp32: 4e-6.
SPREAD = {"bf16": 2.0 ** -9, "f32": 4e-6}
