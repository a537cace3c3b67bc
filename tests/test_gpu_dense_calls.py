"""Calls of the dense operators as programs make them: captured and replayed, on other streams, from threads, beside
one another, with a workspace of the caller's, on either path; results past 32-bit offsets."""
import threading

import pytest
import torch

import dense_cases as dc

pytestmark = pytest.mark.gpu


class Calls:
    """Forward and gradient of a linear layer and of a norm behind it."""

    def __init__(self, lib, M, K, N, act, dt, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed + M)
        t = dc.TORCH[dt]
        Z = 2 * N if act == "swiglu" else N

        def normal(*shape, by=1.0):
            return torch.randn(shape, generator=g, device="cuda").mul_(by).to(t)

        self.lib, self.act = lib, act
        self.x, self.w, self.b, self.r = normal(M, K), normal(Z, K, by=K ** -0.5), normal(Z), normal(M, N)
        self.dy, self.nw = normal(M, N), normal(N)

    def __call__(self):
        y, z = self.lib.sa_linear_fwd(self.x, self.w, self.b, self.act, self.r, want_pre=True)
        n, stats = self.lib.sa_layer_norm_fwd(y, self.nw, self.nw, residual=self.r, want_stats=True)
        dy, _, dw, db = self.lib.sa_layer_norm_bwd(self.dy, y, stats, self.nw, residual=self.r)
        return y, z, n, dy, dw, db, *self.lib.sa_linear_bwd(dy, self.x, self.w, z, self.act)


def equal(x, y):
    return all(torch.equal(a, b) for a, b in zip(x, y))


# products of cut tiles, of whole tiles, of few rows, unaligned (copies in the workspace), fp32
SHAPES = [(300, 4096, 520, "gelu", "bf16"), (20000, 128, 512, "swiglu", "bf16"), (7, 1000, 320, "silu", "bf16"),
          (515, 333, 129, "swiglu", "bf16"), (200, 1000, 264, "gelu", "f32")]


@pytest.mark.parametrize("shape", SHAPES)
def test_a_graph_s_workspace_is_its_own(cuda_lib, shape):
    small, large = Calls(cuda_lib, *shape), Calls(cuda_lib, 3000, 2048, 1536, "swiglu", "f32")
    ref, ref_large = small(), large()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            got = small()
        assert equal(large(), ref_large)
    torch.cuda.synchronize()
    taken = [torch.full((1 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(50)]
    with torch.cuda.stream(s):
        taken += [torch.full((8 << 20,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(10)]
    torch.cuda.synchronize()
    for _ in range(3):
        for x in got:
            x.zero_()
        graph.replay()
        assert equal(large(), ref_large)  # eager calls beside the replay
        torch.cuda.synchronize()
        assert equal(got, ref) and all(bool((x == 0x5A).all()) for x in taken)


def test_two_graphs_and_new_inputs(cuda_lib):
    a, b = Calls(cuda_lib, *SHAPES[0], seed=1), Calls(cuda_lib, *SHAPES[0], seed=2)
    graphs = []
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for c in (a, b):
            c()
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                out = c()
            graphs.append((g, c, out))
    torch.cuda.synchronize()
    t = torch.cuda.Stream()
    for _ in range(3):
        a.x.mul_(0.5)
        ref = [c() for _, c, _ in graphs]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            graphs[0][0].replay()
        with torch.cuda.stream(t):  # at the same time
            graphs[1][0].replay()
        torch.cuda.synchronize()
        assert all(equal(out, r) for (_, _, out), r in zip(graphs, ref))


def test_threads_on_one_stream(cuda_lib):
    calls = [Calls(cuda_lib, *shape, seed=i) for i, shape in enumerate(SHAPES[:3])]
    refs = [c() for c in calls]
    torch.cuda.synchronize()
    wrong = []

    def work(c, ref):
        for _ in range(20):
            if not equal(c(), ref):
                wrong.append(c)

    threads = [threading.Thread(target=work, args=p) for p in zip(calls, refs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not wrong and cuda_lib.sa_linear_get_device_error() == 0


def test_another_stream(cuda_lib):
    c = Calls(cuda_lib, *SHAPES[1])
    ref = c()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = c()
        assert cuda_lib.sa_linear_get_device_error() == 0
    s.synchronize()
    assert equal(got, ref)


def test_the_caller_s_workspace(cuda_lib):
    b, c = cuda_lib, Calls(cuda_lib, *SHAPES[3])
    ref = c()
    M, K, N, act, dt = SHAPES[3]
    sizes = [b.load().sa_linear_workspace_size(M, N, K, 4, 1, bwd, 7) for bwd in (0, 1)]
    ws = torch.full((max(sizes) + 4096,), 0xFF, dtype=torch.uint8, device="cuda")  # need not be cleared
    y, z = b.sa_linear_fwd(c.x, c.w, c.b, act, c.r, want_pre=True, ws=ws)
    assert b.sa_get_device_error(ws) == 0
    ws.fill_(0xFF)
    got = b.sa_linear_bwd(ref[3], c.x, c.w, z, act, ws=ws)
    assert b.sa_get_device_error(ws) == 0
    assert torch.equal(y, ref[0]) and equal(got, ref[6:]) and bool((ws[max(sizes):] == 0xFF).all())
    with pytest.raises(b.SketchError, match="WORKSPACE"):
        b.sa_linear_fwd(c.x, c.w, ws=ws[:256])
    for bad in (torch.empty(1 << 20, dtype=torch.uint8), ws[::2]):
        with pytest.raises(ValueError, match="ws"):
            b.sa_linear_fwd(c.x, c.w, ws=bad)


def test_the_cache_s_status_is_another(cuda_lib):
    """Calls of one family leave the other's status as it is."""
    b = cuda_lib
    pool = b.sa_cache_alloc(2, 1, 64, 64)
    table = torch.tensor([[0, -1]], dtype=torch.int32, device="cuda")
    K = torch.randn((100, 1, 64), device="cuda")
    b.sa_cache_write(pool, table, K, K, torch.tensor([0, 100], dtype=torch.int32, device="cuda"))
    Calls(b, *SHAPES[0])()
    assert b.sa_cache_get_device_error() == 7 and b.sa_linear_get_device_error() == 0
    b._stream_ws_cache.clear()


@pytest.mark.parametrize("shape", SHAPES)
def test_the_paths_agree(cuda_lib, shape):
    c = Calls(cuda_lib, *shape)
    fast = c()
    cuda_lib.sa_select_path(1)
    try:
        slow = c()
        assert cuda_lib.sa_linear_get_device_error() == 0
    finally:
        cuda_lib.sa_select_path(0)
    for a, b in zip(fast, slow):
        # sums in another order, roundings to the type on either side of a border, dz among them
        assert float((a.double() - b.double()).norm()) <= (6e-3 if shape[4] == "bf16" else 1e-5) * float(b.double().norm())


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", [96, 100, 97])
def test_nothing_but_the_outputs_is_written(cuda_lib, dt, N):
    """Rows and bytes around y, z, dx and dw hold what they held, at widths that end inside tiles."""
    b, t = cuda_lib, dc.TORCH[dt]
    lib, M, K = b.load(), 300, 72
    for act, code in (("gelu", 2), ("swiglu", 4)):
        Z = 2 * N if act == "swiglu" else N
        c = Calls(b, M, K, N, act, dt)
        y, z = b.sa_linear_fwd(c.x, c.w, c.b, act, want_pre=True)
        dx, dw, _ = b.sa_linear_bwd(c.dy, c.x, c.w, z, act)
        pad = 64
        bufs = [torch.full((v.numel() + 2 * pad,), 7.0, dtype=t, device="cuda") for v in (y, z, dx, dw)]
        at = [v[pad:].data_ptr() for v in bufs]
        ws = torch.empty(max(lib.sa_linear_workspace_size(M, N, K, code, b._dt_of(t), i, 7) for i in (0, 1)),
                         dtype=torch.uint8, device="cuda")
        st = torch.cuda.current_stream().cuda_stream
        assert lib.sa_linear_fwd(c.x.data_ptr(), K, c.w.data_ptr(), K, c.b.data_ptr(), None, 0, M, N, K, code, b._dt_of(t),
                                 at[0], at[1], ws.data_ptr(), ws.numel(), st) == 0
        assert lib.sa_linear_bwd(c.dy.data_ptr(), N, c.x.data_ptr(), K, c.w.data_ptr(), K, z.data_ptr(), M, N, K, code,
                                 b._dt_of(t), at[2], at[3], None, ws.data_ptr(), ws.numel(), st) == 0
        for buf, ref in zip(bufs, (y, z, dx, dw)):
            assert torch.equal(buf[pad:-pad], ref.flatten())
            assert bool((buf[:pad] == 7).all()) and bool((buf[-pad:] == 7).all())


def test_results_past_32_bit_offsets(cuda_lib):
    b = cuda_lib
    g = torch.Generator(device="cuda").manual_seed(9)
    M, K, N = 70001, 64, 32768  # 2.3e9 results
    x, w = (torch.randn(s, generator=g, device="cuda").bfloat16() for s in ((M, K), (N, K)))
    y = b.sa_linear_fwd(x, w, activation="relu")
    for rows in (slice(0, 300), slice(65500, 65800), slice(M - 300, M)):
        assert torch.equal(y[rows], b.sa_linear_fwd(x[rows], w, activation="relu"))
    dx, dw, db = b.sa_linear_bwd(y, x, w, y, "relu")  # y stands for z: the same sign
    part = b.sa_linear_bwd(y[-300:], x[-300:], w, y[-300:], "relu", True, False, False)[0]
    assert float((dx[-300:].float() - part.float()).norm()) <= 1e-2 * float(part.float().norm())
    assert torch.isfinite(dw).all() and torch.isfinite(db).all()
    del dx, dw, db, part
    n = 16384
    rows = y.view(-1)[: (M * N // n) * n].view(-1, n)
    got, stats = b.sa_layer_norm_fwd(rows, want_stats=True)
    want, last = b.sa_layer_norm_fwd(rows[-100:], want_stats=True)
    assert torch.equal(got[-100:], want) and torch.equal(stats[-100:], last)
    dx = b.sa_layer_norm_bwd(got, rows, stats, want_params=False)[0]
    assert torch.equal(dx[-100:], b.sa_layer_norm_bwd(want, rows[-100:], last, want_params=False)[0])
