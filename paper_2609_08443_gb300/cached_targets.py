"""Sketches in a 4-bit cache and ranked targets that attend over them, as a server and a
trainer on cache hits use them (paper Sec. 4.1 and 3.4): run

    python -m paper_2609_08443_gb300.cached_targets [--refine LAYERS]

One pass: the histories of a few users are sketched (Sec. 3.1), refined by as many layers as are
asked for (Sec. 3.3; none by default), the sketches enter the cache in 4 bits, a request's candidates attend over their user's sketch, each user's live
history grows by a token and is attended to up to each request's own time, and the
candidates' queries get their gradients.  Prints how far 4 bits are from the fp32 sketch.
"""
from __future__ import annotations

import argparse
import math

import torch

from . import binding as b, refine, workloads as wl


class PagePool:
    """Pages of one cache and who holds them: the bookkeeping a server does on the host."""

    def __init__(self, n_pages: int, users: int, max_tokens: int, H: int, d: int, page: int = 64, device="cuda"):
        self.page = page
        self.pool = b.sa_cache_alloc(n_pages, H, d, page, device)
        self.free = list(range(n_pages))
        self.table = torch.full((users, -(-max_tokens // page)), -1, dtype=torch.int32)
        self.lens = [0] * users

    def grow(self, user: int, tokens: int) -> int:
        """Room for ``tokens`` more rows of ``user``; the position the first of them gets."""
        start = self.lens[user]
        have, need = -(-start // self.page), -(-(start + tokens) // self.page)
        if need > self.table.shape[1] or need - have > len(self.free):
            raise RuntimeError("the cache is full: evict a user first")
        for i in range(have, need):
            self.table[user, i] = self.free.pop()
        self.lens[user] += tokens
        return start

    def evict(self, user: int) -> None:
        self.free += [int(p) for p in self.table[user] if p >= 0]
        self.table[user] = -1
        self.lens[user] = 0

    def on_device(self):
        dev = self.pool.device
        return self.pool, self.table.to(dev), torch.tensor(self.lens, dtype=torch.int32, device=dev)


def offsets(counts, device):
    return torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=device)


def run(lengths=(3000, 1200, 700), H=4, P=256, d=64, candidates=100, seed=0, device="cuda", layers=0):
    """The pass described above, with ``layers`` of refinement; returns what a caller may want to check."""
    spec = wl.custom(lengths, H=H, P=P, d=d, seed=seed, bwd=False)
    t = wl.host_to_torch(spec, wl.make_host(spec), device)
    B, N = len(lengths), t["K"].shape[0]

    # a cache miss: sketch the histories, keep the sketches (keys and values in one) in 4 bits
    sketch = b.sa_sketch(t["K"], t["V"], t["cu_seqlens"], t["Q"])  # [B, H, P, d] fp32
    if layers:
        g = torch.Generator(device=device).manual_seed(seed + 2)
        stack = [refine.random_layer(d, 4 * d, t["V"].dtype, device, g) for _ in range(layers)]
        sketch = refine.sa_refine(sketch, t["V"], t["cu_seqlens"], stack).float()
    sketches = PagePool(B * (P // 64 + 1), B, P, H, d, device=device)
    for u in range(B):
        sketches.grow(u, P)
    pool, table, lens = sketches.on_device()
    b.sa_cache_write(pool, table, sketch, sketch)

    # a hit: a request's candidates attend over the cached sketch, and learn
    g = torch.Generator(device=device).manual_seed(seed + 1)
    scale = 1.0 / (math.sqrt(d) * float(sketch.std()))
    q = torch.randn((B * candidates, H, d), generator=g, device=device).bfloat16().requires_grad_(True)
    cu_q = offsets([candidates] * B, device)
    z = b.sa_cache_attention(q, cu_q, pool, table, lens, scale=scale)
    z.float().square().mean().backward()

    # the live history beside it: prefetched once, then one token a user at a time; a request
    # sees the rows up to its own time
    recent = PagePool(sum(n // 64 + 2 for n in lengths), B, max(lengths) + 64, H, d, device=device)
    start = torch.tensor([recent.grow(u, int(n)) for u, n in enumerate(lengths)], dtype=torch.int32, device=device)
    pool_r, table_r, lens_r = recent.on_device()
    b.sa_cache_write(pool_r, table_r, t["K"], t["V"], t["cu_seqlens"], start=start)
    start = torch.tensor([recent.grow(u, 1) for u in range(B)], dtype=torch.int32, device=device)
    _, table_r, lens_r = recent.on_device()
    last = torch.randn((2, B, H, d), generator=g, device=device).bfloat16()
    b.sa_cache_write(pool_r, table_r, last[0], last[1], offsets([1] * B, device), start=start)
    times = torch.randint(0, min(lengths), (B * candidates,), generator=g, device=device, dtype=torch.int32)
    with torch.no_grad():
        r, lse = b.sa_cache_attn_fwd(q, cu_q, pool_r, table_r, lens_r, kv_end=times, want_lse=True)

    # against dense attention over the fp32 sketch
    with torch.no_grad():
        x = q.float().view(B, candidates, H, d).transpose(1, 2)
        dense = torch.softmax(x @ sketch.transpose(-1, -2) * scale, -1) @ sketch
        dense = dense.transpose(1, 2).reshape(B * candidates, H, d)
        error = float((z.float() - dense).norm() / dense.norm())
    fp32, cached = sketch.numel() * 4, B * P * H * 2 * (d // 2 + d // 16)
    return {"z": z, "dq": q.grad, "recent": r, "lse": lse, "times": times, "error": error, "tokens": N,
            "bytes_fp32": fp32, "bytes_cached": cached, "sketches": sketches, "recents": recent}


def main() -> None:
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--refine", type=int, default=0, metavar="LAYERS", help="refinement layers behind the sketch")
    args = parser.parse_args()
    res = run(layers=args.refine)
    torch.cuda.synchronize()
    print(f"{res['tokens']} history rows sketched, {args.refine} refinement layers; sketches {res['bytes_fp32'] / 1e6:.2f} MB in fp32, "
          f"{res['bytes_cached'] / 1e6:.2f} MB cached as keys and values")
    print(f"attention over the 4-bit sketch against fp32: relative difference {res['error']:.3f}")
    print(f"query gradient norm {float(res['dq'].float().norm()):.3e}; "
          f"requests that saw no history: {int((res['times'] == 0).sum())}")


if __name__ == "__main__":
    main()
