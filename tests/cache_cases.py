"""Shared by the cache tests: ragged caches built by the oracle, the operators' answers in
fp64, and how far a kernel may be off, derived from its roundings."""
from __future__ import annotations

import math

import numpy as np
import torch

from oracle import cache_oracle as co
from paper_2609_08443_gb300 import workloads as wl

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, dt):
    x = np.asarray(x, dtype=np.float32)
    return wl.bf16_bits_to_f64(wl.f32_to_bf16_bits(x)) if dt == "bf16" else x.astype(np.float64)


class Cache:
    """Rows of B users quantised by the oracle and laid into shuffled pages; bytes of
    positions nobody wrote hold 0xFF (scale codes that would read as NaN)."""

    def __init__(self, lens, H, d, page, seed=0, k_std=1.0, v_std=1.0, spare=2):
        rng = np.random.default_rng(seed)
        self.lens, self.H, self.d, self.page = [int(n) for n in lens], H, d, page
        self.k = [rng.standard_normal((H, n, d)) * k_std for n in self.lens]
        self.v = [rng.standard_normal((H, n, d)) * v_std for n in self.lens]
        self.kv = [[co.stored(x) for x in part] for part in (self.k, self.v)]
        pages = [-(-n // page) for n in self.lens]
        self.n_pages = sum(pages) + spare
        order = rng.permutation(self.n_pages)
        self.table = np.full((len(lens), max(1, max(pages))), -1, dtype=np.int32)
        self.pool = np.full((self.n_pages, H, 2, page * (d // 2 + d // 16)), 0xFF, dtype=np.uint8)
        at = 0
        for b, n in enumerate(pages):
            for i in range(n):
                p = self.table[b, i] = order[at]
                at += 1
                rows = slice(i * page, min((i + 1) * page, self.lens[b]))
                m = rows.stop - rows.start
                for h in range(H):
                    for j, src in enumerate((self.k, self.v)):
                        rec = co.record(src[b][h, rows])
                        self.pool[p, h, j, : m * d // 2] = rec[: m * d // 2]
                        self.pool[p, h, j, page * d // 2: page * d // 2 + m * d // 16] = rec[m * d // 2:]

    def tensors(self, device="cuda"):
        return (torch.from_numpy(self.pool).to(device), torch.from_numpy(self.table).to(device),
                torch.tensor(self.lens, dtype=torch.int32, device=device))


def offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def reference(cache, q, n_q, G, scale, begin=None, end=None, dout=None, out=None, lse=None):
    """fp64 (out, lse, and dq if dout is given) for packed queries q [T, H * G, d], with the sums
    that bound a kernel's error: A = sum p |v|, V = sum |v|, S = largest sum |q k| |scale|, W = |scale| sum |ds| |k|,
    U = |scale| sum p |k| sum |dout v|."""
    T, Hq, d = q.shape
    r = {k: np.zeros((T, Hq, d)) for k in ("out", "dq", "A", "V", "W", "U")}
    r["lse"], r["S"] = np.full((T, Hq), -np.inf), np.zeros((T, Hq))
    cu = offsets(n_q)
    for b, n in enumerate(n_q):
        rows = range(int(cu[b]), int(cu[b + 1]))
        win = [co.window(t, cache.lens[b], begin, end) for t in rows]
        for h in range(Hq):
            k, v = cache.kv[0][b][h // G], cache.kv[1][b][h // G]
            sl = (slice(int(cu[b]), int(cu[b + 1])), h)
            o, l = co.attention(q[sl], k, v, scale, win)
            r["out"][sl], r["lse"][sl] = o, l
            if dout is not None:
                o, l = (o, l) if out is None else (out[sl], lse[sl])
                r["dq"][sl] = co.attention_grad(q[sl], k, v, scale, win, o, l, dout[sl])
            for i, (lo, hi) in enumerate(win):
                if lo >= hi:
                    continue
                t = int(cu[b]) + i
                r["S"][t, h] = abs(scale) * (np.abs(k[lo:hi]) @ np.abs(q[t, h])).max()
                p = np.exp(scale * (k[lo:hi] @ q[t, h]) - r["lse"][t, h])
                r["A"][t, h] = p @ np.abs(v[lo:hi])
                r["V"][t, h] = np.abs(v[lo:hi]).sum(0)
                if dout is not None:
                    do, ou = dout[t, h], (r["out"] if out is None else out)[t, h]
                    ds = p * (v[lo:hi] @ do - ou @ do)
                    dp = np.abs(v[lo:hi]) @ np.abs(do) + np.abs(ou) @ np.abs(do)
                    r["W"][t, h] = abs(scale) * (np.abs(ds) @ np.abs(k[lo:hi]))
                    r["U"][t, h] = abs(scale) * ((p * dp) @ np.abs(k[lo:hi]))
    return r


def limits(r, d, dt, L):
    """Element-wise error bounds of (out, lse, dq).

    u = 2^-23 a rounding or truncation of an fp32 accumulation.  A score is a sum of d products
    (three bf16 terms each for fp32), so it is off by at most e_s = (d + 8) u S; its multiplication by
    log2 e, the shift and 2^x add a few u (|S| + 1).  Weights are rounded to float16 (2^-11 each way at
    most; two terms leave 2^-21; either way a weight below 2^-37 of the largest, half of float16's
    smallest number after the kernel's lift by 2^12, is lost whole), their products summed in fp32 over L / 16 steps.  The result is
    rounded to its type once."""
    u = 2.0 ** -23
    e_s = (d + 8) * u * r["S"] + 8 * u * (r["S"] + 1 + np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)))
    e_p = 2 * e_s + 4 * u
    e_sum = (L / 16 + 16) * u
    e_w = 2.0 ** -11 if dt == "bf16" else 2.0 ** -21
    e_r = 2.0 ** -8 if dt == "bf16" else u
    out = r["A"] * (e_p + e_w + e_sum)[..., None] + r["V"] * 2.0 ** -37 + e_r * np.abs(r["out"])
    lse = e_s + e_sum + 8 * u * np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)) + 1e-12
    # weights enter ds times dout . v - D, itself off by (2 d + 8) u of its absolute sums
    e_ds = 2.0 ** -8 if dt == "bf16" else 2.0 ** -22
    dq = r["W"] * (e_p + e_ds + e_sum)[..., None] + r["U"] * ((2 * d + 16) * u + e_sum) + e_r * np.abs(r["dq"])
    return out, lse, dq


def check(name, got, ref, most):
    got = got.detach().double().cpu().numpy() if torch.is_tensor(got) else np.asarray(got)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    inf = ~np.isfinite(ref)
    assert np.array_equal(got[inf], ref[inf]), f"{name}: infinities differ"
    assert np.all(np.isfinite(got[~inf])), f"{name}: not finite"
    over = np.abs(got[~inf] - ref[~inf]) - (most[~inf] + 1e-30)
    assert not np.any(over > 0), f"{name}: {int(np.sum(over > 0))} of {over.size} off by more than allowed, worst by {over.max():.3e}"


def queries(T, Hq, d, dt, seed, std=1.0):
    rng = np.random.default_rng(1000 + seed)
    return rounded(rng.standard_normal((T, Hq, d)) * std, dt)


def to_gpu(x, dt):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", torch.float32).to(TORCH[dt])


def default_scale(d):
    return float(np.float32(1.0 / math.sqrt(d)))
