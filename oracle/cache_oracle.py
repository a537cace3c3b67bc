"""fp64 NumPy reference of the 4-bit cache: the stored values of a row, the bytes of a
page, and attention over cached rows with the gradient of its queries.

Written from the definitions in ``include/sa_cache.h`` and shares no code with the
CUDA path.  A row of width d is cut into groups of 16 features; a group is stored as a
scale s = (8 + m) 2^(e - 18) (code 8 e + m in 8..225, the smallest with 7.5 s >= max |x|)
and 16 levels, the whole numbers nearest to x / s (halves towards zero, at most 7).
"""
from __future__ import annotations

import numpy as np

GROUP = 16
CODES = np.arange(8, 226)
SCALES = (8 + CODES % 8) * np.exp2(CODES // 8 - 18.0)


def quantise(x):
    """(levels, codes) of fp64 rows [..., d]: whole numbers [..., d], scale codes [..., d/16]."""
    x = np.asarray(x, dtype=np.float64)
    x = np.where(np.isnan(x), 0.0, x).reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    a = np.abs(x)
    i = np.minimum(np.searchsorted(7.5 * SCALES, a.max(-1)), CODES.size - 1)
    s = SCALES[i][..., None]
    # thresholds (k + 1/2) s are exact in fp64: count the ones below |x|
    level = sum((a > (k + 0.5) * s).astype(np.float64) for k in range(7))
    level = np.where(np.signbit(x), -level, level)
    return level.reshape(*x.shape[:-2], x.shape[-2] * GROUP), CODES[i]


def stored(x):
    """The values rows [..., d] read back as."""
    level, code = quantise(x)
    s = (8 + code % 8) * np.exp2(code // 8 - 18.0)
    return level * np.repeat(s, GROUP, axis=-1)


# the feature at nibble n of a 32-bit word (lowest first)
NIBBLES = (0, 2, 4, 6, 1, 3, 5, 7)


def record(x):
    """The bytes of one record for a page of rows x [page, d]."""
    level, code = quantise(x)
    page, d = level.shape
    u = (level + 8).astype(np.uint32).reshape(page, d // 8, 8)
    word = np.zeros((page, d // 8), dtype=np.uint32)
    for n, f in enumerate(NIBBLES):
        word |= u[..., f] << np.uint32(4 * n)
    codes = np.stack([(word >> np.uint32(8 * i)) & np.uint32(255) for i in range(4)], -1).astype(np.uint8)
    return np.concatenate([codes.reshape(-1), code.astype(np.uint8).reshape(-1)])


def window(t, length, begin, end):
    lo = 0 if begin is None else max(0, int(begin[t]))
    hi = length if end is None else min(length, int(end[t]))
    return lo, max(lo, hi)


def attention(q, k, v, scale, windows):
    """(out [R, d], lse [R]) of queries q over one user's and head's rows k, v [L, d]; query r sees windows[r]."""
    R, d = q.shape
    out, lse = np.zeros((R, d)), np.full(R, -np.inf)
    for r, (lo, hi) in enumerate(windows):
        if lo >= hi:
            continue
        s = scale * (k[lo:hi] @ q[r])
        m = s.max()
        p = np.exp(s - m)
        z = p.sum()
        out[r] = (p @ v[lo:hi]) / z
        lse[r] = m + np.log(z)
    return out, lse


def attention_grad(q, k, v, scale, windows, out, lse, dout):
    """dq [R, d] for the gradient dout; out and lse as the forward gave them."""
    dq = np.zeros(q.shape)
    for r, (lo, hi) in enumerate(windows):
        if lo >= hi:
            continue
        p = np.exp(scale * (k[lo:hi] @ q[r]) - lse[r])
        ds = p * (v[lo:hi] @ dout[r] - out[r] @ dout[r])
        dq[r] = scale * (ds @ k[lo:hi])
    return dq
