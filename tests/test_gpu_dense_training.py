"""Training steps through the differentiable forms as programs run them: captured and replayed, from threads, on rows that
overlap or repeat, and with a workspace that is not kept."""
import threading

import pytest
import torch

import dense_sums as ds

pytestmark = pytest.mark.gpu


class Net:
    """norm(x + feed-forward(x)) with gradients of everything"""

    def __init__(self, lib, rows=500, d=128, F=256, dt=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def leaf(*s, by=1.0):
            return torch.randn(s, generator=g, device="cuda").mul_(by).to(dt).requires_grad_(True)

        self.lib, self.x = lib, leaf(rows, d)
        self.w_in, self.b_in, self.w_out = leaf(2 * F, d, by=d ** -0.5), leaf(2 * F), leaf(d, F, by=F ** -0.5)
        self.nw, self.nb = leaf(d), leaf(d)
        self.dy = torch.randn((rows, d), generator=g, device="cuda").to(dt)

    def leaves(self):
        return self.x, self.w_in, self.b_in, self.w_out, self.nw, self.nb

    def step(self):
        b = self.lib
        hidden = b.sa_linear(self.x, self.w_in, self.b_in, "swiglu")
        y = b.sa_layer_norm(b.sa_linear(hidden, self.w_out, residual=self.x), self.nw, self.nb)
        return y.detach(), *torch.autograd.grad(y, self.leaves(), self.dy)


def equal(a, b):
    return all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("rows,dt", [(500, torch.bfloat16), (7, torch.bfloat16), (300, torch.float32), (9, torch.float32)])
def test_a_captured_step(cuda_lib, rows, dt):
    """Forward and gradients in one graph, replayed on other inputs and on another stream than it was captured on."""
    net = Net(cuda_lib, rows=rows, dt=dt)
    s, t = torch.cuda.Stream(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        net.step()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            got = net.step()
    torch.cuda.synchronize()
    for i in range(3):
        with torch.no_grad():
            net.x.copy_(torch.randn(net.x.shape, device="cuda"))
            net.w_in.mul_(0.9)
        ref = net.step()
        torch.cuda.synchronize()
        with torch.cuda.stream((s, t, torch.cuda.current_stream())[i]):
            graph.replay()
        torch.cuda.synchronize()
        assert equal(got, ref)


def test_steps_of_two_threads(cuda_lib):
    nets = [Net(cuda_lib, rows=r, seed=r) for r in (400, 3000)]
    refs = [n.step() for n in nets]
    torch.cuda.synchronize()
    wrong = []

    def work(net, ref):
        wrong.extend(net for _ in range(15) if not equal(net.step(), ref))

    threads = [threading.Thread(target=work, args=p) for p in zip(nets, refs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_gradients_that_accumulate(cuda_lib):
    """The same leaf as input and residual, and two passes into .grad."""
    b = cuda_lib
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((60, 64), generator=g, device="cuda", requires_grad=True)
    w = torch.randn((64, 64), generator=g, device="cuda").mul_(0.1).requires_grad_(True)
    n = torch.randn(64, generator=g, device="cuda", requires_grad=True)
    dy = torch.randn((60, 64), generator=g, device="cuda")
    for _ in range(2):
        b.sa_layer_norm(b.sa_linear(x, w, activation="gelu", residual=x), n, residual=x).backward(dy)
    x64, w64, n64 = (v.detach().double().requires_grad_() for v in (x, w, n))
    f = torch.nn.functional
    f.layer_norm(f.gelu(x64 @ w64.T) + 2 * x64, (64,), n64).backward(2 * dy.double())
    for p, q in ((x, x64), (w, w64), (n, n64)):
        assert ds.spread(p.grad, q.grad) <= 1e-5


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M", [9, 200])
def test_rows_that_overlap_or_repeat(cuda_lib, M, dt):
    """Windows of a longer row as x, one row as all of W's, and dy of one row."""
    b, t = cuda_lib, {"bf16": torch.bfloat16, "f32": torch.float32}[dt]
    K, N = 96, 64
    g = torch.Generator(device="cuda").manual_seed(M)
    line = torch.randn(M * 8 + K, generator=g, device="cuda").to(t)
    w = torch.randn((N, K), generator=g, device="cuda").mul_(0.1).to(t)
    dy = torch.randn((M, N), generator=g, device="cuda").to(t)
    for step in (1, 5, 8):
        x = line.as_strided((M, K), (step, 1))
        for w_ in (w, w[:1].expand(N, K)):
            assert torch.equal(b.sa_linear_fwd(x, w_, activation="silu"), b.sa_linear_fwd(x.contiguous(), w_.contiguous(), activation="silu"))
            for dy_ in (dy, dy[:1].expand(M, N)):
                got = b.sa_linear_bwd(dy_, x, w_)
                x64, w64, dy64 = (v.double() for v in (x, w_, dy_))
                for v, ref in zip(got, (dy64 @ w64, dy64.T @ x64, dy64.sum(0))):
                    assert ds.spread(v, ref) <= 1.2 * ds.SPREAD[dt]
        y, stats = b.sa_layer_norm_fwd(x, want_stats=True)
        ref = ds.norm_reference(x.double(), None, torch.ones(K, device="cuda").double(), torch.zeros(K, device="cuda").double(),
                                x.double(), 1e-5, 152)
        ds.check("y", y, *ref["y"])
        dx, _, dw, db = b.sa_layer_norm_bwd(x, x, stats)
        for name, v, of in (("dx", dx, "dh"), ("dw", dw, "dw"), ("db", db, "db")):
            ds.check(name, v, *ref[of])


def test_a_large_workspace_s_status_can_be_read(cuda_lib):
    """It is not kept by the thread, but until the stream's next call."""
    b = cuda_lib
    x = torch.randn((40000, 512), device="cuda").bfloat16()
    w = torch.randn((1024, 512), device="cuda").bfloat16()
    y, z = b.sa_linear_fwd(x, w, activation="gelu", want_pre=True)
    first = b.sa_linear_bwd(y, x, w, z, "gelu")
    assert b._linear_workspace_size(0, 40000, 1024, 512, 2, 1, 1, 0) > b._DENSE_KEPT
    assert b.sa_linear_get_device_error() == 0
    for _ in range(5):  # memory that comes and goes
        junk = torch.full((100 << 20,), 0x5A, dtype=torch.uint8, device="cuda")
        del junk
        assert equal(b.sa_linear_bwd(y, x, w, z, "gelu"), first)
    assert b.sa_linear_get_device_error() == 0
