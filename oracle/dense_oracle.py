"""fp64 NumPy reference of layer norm (of a sum) and of linear layers with bias, activation and
residual, with their gradients.  Rows are 2-D here: [rows, features]."""
from __future__ import annotations

import math

import numpy as np

ACTIVATIONS = ("none", "relu", "gelu", "silu", "swiglu")


def layer_norm(h, w, b, eps):
    """(y, mean, rstd) for rows h = x + r."""
    h = np.asarray(h, dtype=np.float64)
    mean = h.mean(1)
    var = ((h - mean[:, None]) ** 2).mean(1)
    rstd = 1.0 / np.sqrt(var + eps)
    return (h - mean[:, None]) * rstd[:, None] * w + b, mean, rstd


def layer_norm_grad(dy, h, w, eps):
    """(dh, dw, db): the chain rule through mean and variance."""
    _, mean, rstd = layer_norm(h, 1.0, 0.0, eps)
    xh = (h - mean[:, None]) * rstd[:, None]
    g = dy * w
    dh = rstd[:, None] * (g - g.mean(1, keepdims=True) - xh * (g * xh).mean(1, keepdims=True))
    return dh, (dy * xh).sum(0), dy.sum(0)


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def sigmoid(z):
    return np.where(z >= 0, 1 / (1 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1 + np.exp(-np.abs(z))))


def activate(z, act):
    if act == "none":
        return z
    if act == "relu":
        return np.maximum(z, 0)
    if act == "gelu":
        return z * _erfc(-z / math.sqrt(2)) / 2
    if act == "silu":
        return z * sigmoid(z)
    n = z.shape[1] // 2
    return z[:, :n] * sigmoid(z[:, :n]) * z[:, n:]


def activation_grad(dy, z, act):
    if act == "none":
        return dy
    if act == "relu":
        return np.where(z > 0, dy, 0)
    if act == "gelu":
        return dy * (_erfc(-z / math.sqrt(2)) / 2 + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi))
    if act == "silu":
        p = sigmoid(z)
        return dy * (p + z * p * (1 - p))
    n = z.shape[1] // 2
    a, u = z[:, :n], z[:, n:]
    p = sigmoid(a)
    return np.concatenate([dy * u * (p + a * p * (1 - p)), dy * a * p], 1)


def linear(x, w, b, r, act):
    """(y, z)"""
    z = x @ w.T + (0 if b is None else b)
    return activate(z, act) + (0 if r is None else r), z


def linear_grad(dy, x, w, z, act):
    """(dx, dw, db, dz) for the forward's z"""
    dz = activation_grad(dy, z, act)
    return dz @ w, dz.T @ x, dz.sum(0), dz
