"""Layer norm and linear layers on the GPU against the fp64 reference, element by element."""
import numpy as np
import pytest
import torch

import dense_cases as dc
from oracle import dense_oracle as do

pytestmark = pytest.mark.gpu

EPS = 1e-5
WIDTHS = [1, 2, 7, 8, 63, 64, 65, 128, 129, 200, 256, 257, 511, 512, 513, 1024, 1025, 2048, 2056, 4096, 4097, 8192,
          8200, 16384, 16383]


def norm_call(b, c, x="bf16", r=None, y="bf16"):
    t = {k: dc.to_gpu(c[k], dt) for k, dt in (("x", x), ("r", r), ("w", y), ("b", y), ("dy", y)) if c[k] is not None}
    t.setdefault("r", None)
    out, stats = b.sa_layer_norm_fwd(t["x"], t["w"], t["b"], t["r"], EPS, dc.TORCH[y], want_stats=True)
    dx, dr, dw, db = b.sa_layer_norm_bwd(t["dy"], t["x"], stats, t["w"], t["r"])
    return out, stats, dx, dr, dw, db


def norm_check(b, rows, n, seed, x="bf16", r=None, y="bf16", offset=0.5):
    c = dc.norm_inputs(rows, n, seed, x, r, y, offset)
    out, stats, dx, dr, dw, db = norm_call(b, c, x, r, y)
    (y64, e_y), (mean, e_m), (rstd, e_r) = dc.norm_limits(c, EPS, y)
    dc.check("y", out, y64, e_y)
    dc.check("mean", stats[:, 0], mean, e_m)
    dc.check("rstd", stats[:, 1], rstd, e_r)
    (dh, e_dh), (gw, e_gw), (gb, e_gb) = dc.norm_grad_limits(c, EPS, x, r, y)
    dc.check("dx", dx, dh, e_dh + dc.half_step(x) * (np.abs(dh) + e_dh))
    if r is not None:
        dc.check("dr", dr, dh, e_dh + dc.half_step(r) * (np.abs(dh) + e_dh))
        assert (dr is dx) == (r == x)
    dc.check("dw", dw, gw, e_gw)
    dc.check("db", db, gb, e_gb)


@pytest.mark.parametrize("n", WIDTHS)
def test_norm_widths(cuda_lib, n):
    norm_check(cuda_lib, 37, n, n)


@pytest.mark.parametrize("rows", [1, 2, 15, 16, 17, 33, 1000, 5001])
@pytest.mark.parametrize("n", [64, 128, 200])
def test_norm_rows(cuda_lib, rows, n):
    norm_check(cuda_lib, rows, n, rows + n, "f32", "bf16", "bf16")


@pytest.mark.parametrize("x", ["bf16", "f32"])
@pytest.mark.parametrize("r", [None, "bf16", "f32"])
@pytest.mark.parametrize("y", ["bf16", "f32"])
@pytest.mark.parametrize("n", [128, 333, 1024, 12000])
def test_norm_types(cuda_lib, x, r, y, n):
    norm_check(cuda_lib, 19, n, n, x, r, y)


def test_norm_far_from_zero(cuda_lib):
    """A mean far above the deviations costs the digits of h itself, none of the variance's."""
    norm_check(cuda_lib, 50, 768, 1, "f32", None, "f32", offset=1000.0)


def test_norm_many_rows(cuda_lib):
    norm_check(cuda_lib, 40013, 128, 5, "f32", "bf16", "bf16")


def test_norm_constant_rows(cuda_lib):
    """No variance: y is the bias, the gradient stays finite."""
    c = dc.norm_inputs(5, 96, 1, "f32", None, "f32")
    c["x"][:] = 2.5
    out, stats, dx, _, _, _ = norm_call(cuda_lib, c, "f32", None, "f32")
    assert torch.equal(out.cpu().double(), torch.from_numpy(np.broadcast_to(c["b"], (5, 96)).copy()))
    assert torch.isfinite(dx).all() and torch.allclose(stats[:, 1], torch.tensor(EPS ** -0.5, device="cuda"))


def test_norm_without_parameters(cuda_lib):
    c = dc.norm_inputs(9, 160, 2, "bf16", None, "bf16")
    c["w"], c["b"] = np.ones(160), np.zeros(160)
    x, dy = dc.to_gpu(c["x"], "bf16"), dc.to_gpu(c["dy"], "bf16")
    out, stats = cuda_lib.sa_layer_norm_fwd(x, eps=EPS, want_stats=True)
    dx, dr, dw, db = cuda_lib.sa_layer_norm_bwd(dy, x, stats)
    (y64, e), _, _ = dc.norm_limits(c, EPS, "bf16")
    dc.check("y", out, y64, e)
    (dh, e), (gw, e_gw), (gb, e_gb) = dc.norm_grad_limits(c, EPS, "bf16", None, "f32")
    dc.check("dx", dx, dh, e + dc.half_step("bf16") * (np.abs(dh) + e))
    assert dr is None and dw.dtype is torch.float32
    dc.check("dw", dw, gw, e_gw)
    dc.check("db", db, gb, e_gb)


def test_norm_rows_do_not_mix(cuda_lib):
    """A NaN or an infinity stays in its row."""
    c = dc.norm_inputs(40, 128, 3, "f32", None, "f32")
    clean = norm_call(cuda_lib, c, "f32", None, "f32")
    c["x"][7, 5], c["x"][21, 0] = np.nan, np.inf
    out, stats, dx, _, _, _ = norm_call(cuda_lib, c, "f32", None, "f32")
    keep = [i for i in range(40) if i not in (7, 21)]
    for a, b in ((out, clean[0]), (stats, clean[1]), (dx, clean[2])):
        assert torch.equal(a[keep], b[keep]) and not torch.isfinite(a[[7, 21]]).all(-1).any()


@pytest.mark.parametrize("n", [128, 130, 1024])
def test_norm_strides(cuda_lib, n):
    """Columns of a wider tensor, every second row, rows of a 4-d tensor, repeated rows."""
    b = cuda_lib
    g = torch.Generator(device="cuda").manual_seed(n)
    wide = torch.randn((12, 2, n + 21), generator=g, device="cuda").bfloat16()
    w = torch.randn(n, generator=g, device="cuda").bfloat16()
    for x in (wide[:, 1, 5:5 + n], wide[::2, 0, :n], wide[:, :, 8:8 + n], wide[3:4, :, 2:2 + n],
              wide[0, 0, :n].expand(6, n)):
        y, stats = b.sa_layer_norm_fwd(x, w, want_stats=True)
        y2, stats2 = b.sa_layer_norm_fwd(x.contiguous(), w, want_stats=True)
        # sums over a row are taken in another order where rows are not aligned: a step of bf16 in y at most
        assert y.shape == x.shape and torch.allclose(y.float(), y2.float(), rtol=2 ** -7, atol=1e-5)
        assert torch.allclose(stats, stats2, rtol=1e-5, atol=1e-6)
        dx, _, dw, db = b.sa_layer_norm_bwd(x, x, stats, w)
        dx2, _, dw2, db2 = b.sa_layer_norm_bwd(x.contiguous(), x.contiguous(), stats, w)
        assert torch.allclose(dx.float(), dx2.float(), rtol=2e-2, atol=1e-3)
        assert torch.allclose(dw.float(), dw2.float(), rtol=2e-2, atol=1e-2)


def test_norm_refuses_uneven_rows(cuda_lib):
    x = torch.randn((4, 3, 64), device="cuda")
    for bad in (x[:, :2], x.transpose(1, 2)):
        with pytest.raises(ValueError, match="rows"):
            cuda_lib.sa_layer_norm_fwd(bad)


def test_norm_in_place(cuda_lib):
    x = torch.randn((70, 256), device="cuda")
    want = cuda_lib.sa_layer_norm_fwd(x)
    lib = cuda_lib.load()
    st = lib.sa_layer_norm_fwd(x.data_ptr(), 256, 0, None, 0, 0, None, None, 0, 70, 256, 1e-5, x.data_ptr(), 0, None,
                               torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(x, want)


def test_norm_rows_behind_are_left(cuda_lib):
    buf = torch.full((20, 128), 7.0, device="cuda")
    lib = cuda_lib.load()
    x = torch.randn((11, 128), device="cuda")
    st = lib.sa_layer_norm_fwd(x.data_ptr(), 128, 0, None, 0, 0, None, None, 0, 11, 128, 1e-5, buf.data_ptr(), 0, None,
                               torch.cuda.current_stream().cuda_stream)
    assert st == 0 and torch.equal(buf[11:], torch.full((9, 128), 7.0, device="cuda"))


def test_norm_no_rows(cuda_lib):
    x = torch.empty((0, 64), device="cuda")
    y, stats = cuda_lib.sa_layer_norm_fwd(x, want_stats=True)
    dx, _, dw, db = cuda_lib.sa_layer_norm_bwd(x, x, stats)
    assert y.shape == (0, 64) and dx.shape == (0, 64) and not dw.any() and not db.any()


def test_norm_autograd(cuda_lib):
    g = torch.Generator().manual_seed(0)
    x, r = (torch.randn((3, 4, 96), generator=g, dtype=torch.float64) for _ in range(2))
    w, bias, dy = torch.randn(96, generator=g).double(), torch.randn(96, generator=g).double(), torch.randn((3, 4, 96), generator=g).double()
    leaves = [t.float().cuda().requires_grad_() for t in (x, w, bias, r)]
    cuda_lib.sa_layer_norm(*leaves).backward(dy.float().cuda())
    ref = [t.requires_grad_() for t in (x, w, bias, r)]
    torch.nn.functional.layer_norm(ref[0] + ref[3], (96,), ref[1], ref[2], 1e-5).backward(dy)
    for a, b in zip(leaves, ref):
        assert torch.allclose(a.grad.cpu().double(), b.grad, rtol=1e-4, atol=1e-4)
    assert leaves[0].grad.data_ptr() != leaves[3].grad.data_ptr()
    frozen = [leaves[0].detach(), leaves[1], leaves[2].detach(), leaves[3].detach()]
    leaves[1].grad = None
    cuda_lib.sa_layer_norm(*frozen).sum().backward()
    assert leaves[1].grad is not None
    y = cuda_lib.sa_layer_norm(leaves[0], leaves[1])
    dx, = torch.autograd.grad(y.square().sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


# ----------------------------------------------------------------- linear

def linear_call(b, c, act, dt, z=None):
    """Forward, and the gradient for the forward's own z."""
    t = {k: dc.to_gpu(v, dt) for k, v in c.items()}
    y, pre = b.sa_linear_fwd(t["x"], t["w"], t["b"], act, t["r"], want_pre=True)
    dx, dw, db = b.sa_linear_bwd(t["dy"], t["x"], t["w"], pre, act)
    return y, pre, dx, dw, db


def linear_check(b, M, K, N, act, dt, seed=0, **kw):
    c = dc.linear_inputs(M, K, N, act, dt, seed + 7 * M + K + N, **kw)
    y, pre, dx, dw, db = linear_call(b, c, act, dt)
    assert b.sa_linear_get_device_error() == 0
    (y64, e_y), (z64, e_z) = dc.linear_limits(c, act, dt)
    dc.check("y", y, y64, e_y)
    if act == "none":
        assert pre is None
        z = z64
    else:
        dc.check("z", pre, z64, e_z)
        z = pre.double().cpu().numpy()
    for name, got, (ref, e) in zip(("dx", "dw", "db"), (dx, dw, db), dc.linear_grad_limits(c, z, act, dt)):
        dc.check(name, got, ref, e)


SHAPES = [(1, 1, 1), (1, 64, 128), (3, 17, 5), (64, 64, 64), (128, 128, 128), (129, 65, 130), (255, 100, 257),
          (256, 256, 512), (300, 520, 300), (1000, 72, 40), (5, 1000, 700), (40, 16, 1100), (16, 2048, 320),
          (33, 4100, 36)]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", do.ACTIVATIONS)
@pytest.mark.parametrize("shape", SHAPES)
def test_linear(cuda_lib, shape, act, dt):
    linear_check(cuda_lib, *shape, act, dt, bias=True, res=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 2, 7, 8, 9, 16, 17, 31, 32, 33, 64, 65, 127])
@pytest.mark.parametrize("act", ["none", "swiglu"])
def test_linear_few_rows(cuda_lib, M, act, dt):
    linear_check(cuda_lib, M, 512, 384, act, dt, bias=False, res=False)
    linear_check(cuda_lib, M, 331, 250, act, dt, bias=True, res=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(5000, 128, 512), (20011, 128, 128), (2048, 1024, 1024), (700, 2000, 1500)])
def test_linear_larger(cuda_lib, shape, dt):
    """Against 64 bits on the GPU, norm-wise: bf16 results are off by their own rounding (and dz's), fp32 by sums."""
    b = cuda_lib
    M, K, N = shape
    g = torch.Generator(device="cuda").manual_seed(M)
    t = {k: torch.randn(s, generator=g, device="cuda").mul_(f).to(dc.TORCH[dt]) for k, s, f in (
        ("x", (M, K), 1), ("w", (2 * N, K), K ** -0.5), ("b", (2 * N,), 0.3), ("dy", (M, N), 1))}
    y, z = b.sa_linear_fwd(t["x"], t["w"], t["b"], "swiglu", want_pre=True)
    dx, dw, db = b.sa_linear_bwd(t["dy"], t["x"], t["w"], z, "swiglu")
    x, w, bias, dy = (t[k].double() for k in ("x", "w", "b", "dy"))
    zr = x @ w.T + bias
    z64 = z.double().requires_grad_()
    torch.autograd.backward(torch.nn.functional.silu(z64[:, :N]) * z64[:, N:], dy)
    dz = z64.grad
    ref = {"y": torch.nn.functional.silu(zr[:, :N]) * zr[:, N:], "z": zr, "dx": dz @ w, "dw": dz.T @ x, "db": dz.sum(0)}
    # a rounding spreads evenly over its step: 2^-9 / sqrt(3) of bf16, twice where dz is an operand; sums of fp32 4e-6
    most = 2.0 ** -9 if dt == "bf16" else 4e-6
    for k, got in (("y", y), ("z", z), ("dx", dx), ("dw", dw), ("db", db)):
        off = float((got.double() - ref[k]).norm() / ref[k].norm())
        assert off <= most * (1.5 if k in ("dx", "dw") else 1), (k, off)


@pytest.mark.parametrize("act", do.ACTIVATIONS)
@pytest.mark.parametrize("shape", [(5000, 72, 520), (5000, 130, 519), (20000, 16, 40), (2500, 200, 1100)])
def test_linear_many_tiles(cuda_lib, shape, act):
    """Several tiles, and chunks of them, for each of the warps that end them."""
    linear_check(cuda_lib, *shape, act, "bf16", bias=True, res=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_large_values(cuda_lib, dt):
    """Activations far out on both sides."""
    for act in do.ACTIVATIONS:
        linear_check(cuda_lib, 60, 96, 80, act, dt, bias=True, scale=12.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_strides(cuda_lib, dt):
    """Operands cut out of wider tensors at any offset give the same bits as contiguous ones."""
    b, t = cuda_lib, dc.TORCH[dt]
    g = torch.Generator(device="cuda").manual_seed(4)
    M, K, N = 150, 136, 72
    wide = torch.randn((M, K + 30), generator=g, device="cuda").to(t)
    ww = torch.randn((N, 2 * K), generator=g, device="cuda").to(t)
    rw = torch.randn((M, N + 5), generator=g, device="cuda").to(t)
    bias = torch.randn(N, generator=g, device="cuda").to(t)
    for ox, ow, orr in ((0, 0, 0), (8, 16, 1), (3, 5, 2), (1, 8, 5), (16, 1, 3)):
        x, w, r = wide[:, ox:ox + K], ww[:, ow:ow + K], rw[:, orr:orr + N]
        y, z = b.sa_linear_fwd(x, w, bias, "silu", r, want_pre=True)
        y2, z2 = b.sa_linear_fwd(x.contiguous(), w.contiguous(), bias, "silu", r.contiguous(), want_pre=True)
        assert torch.equal(y, y2) and torch.equal(z, z2)
        got = b.sa_linear_bwd(r, x, w, z, "silu")
        want = b.sa_linear_bwd(r.contiguous(), x.contiguous(), w.contiguous(), z, "silu")
        assert torch.allclose(got[2].float(), want[2].float(), rtol=1e-2, atol=1e-3)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    row = wide[:1, :K].expand(9, K)  # repeated rows
    assert torch.equal(b.sa_linear_fwd(row, ww[:, :K]), b.sa_linear_fwd(row.contiguous(), ww[:, :K]))
    x4 = torch.randn((3, 4, 5, 64), generator=g, device="cuda").to(t)
    w4 = torch.randn((24, 64), generator=g, device="cuda").to(t)
    assert torch.equal(b.sa_linear_fwd(x4, w4), b.sa_linear_fwd(x4.reshape(60, 64), w4).view(3, 4, 5, 24))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_what_is_wanted(cuda_lib, dt):
    b = cuda_lib
    c = dc.linear_inputs(70, 90, 48, "gelu", dt, 1)
    t = {k: dc.to_gpu(v, dt) for k, v in c.items()}
    _, z = b.sa_linear_fwd(t["x"], t["w"], t["b"], "gelu", want_pre=True)
    whole = b.sa_linear_bwd(t["dy"], t["x"], t["w"], z, "gelu")
    for want in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 0, 0)):
        part = b.sa_linear_bwd(t["dy"], t["x"], t["w"], z, "gelu", *map(bool, want))
        for got, ref, on in zip(part, whole, want):
            assert torch.equal(got, ref) if on else got is None


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_no_rows(cuda_lib, dt):
    t = dc.TORCH[dt]
    x, w = torch.empty((0, 32), dtype=t, device="cuda"), torch.randn((16, 32), device="cuda").to(t)
    y, z = cuda_lib.sa_linear_fwd(x, w, activation="relu", want_pre=True)
    assert y.shape == (0, 16) and z.shape == (0, 16)
    dx, dw, db = cuda_lib.sa_linear_bwd(y, x, w, z, "relu")
    assert dx.shape == (0, 32) and not dw.any() and not db.any()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_rows_do_not_mix(cuda_lib, dt):
    """A NaN stays in its row of y, z and dx."""
    c = dc.linear_inputs(200, 128, 96, "silu", dt, 8)
    clean = linear_call(cuda_lib, c, "silu", dt)
    c["x"][130, 7] = np.nan
    dirty = linear_call(cuda_lib, c, "silu", dt)
    keep = torch.arange(200) != 130
    for i in (0, 1, 2):
        assert torch.equal(clean[i][keep], dirty[i][keep]) and torch.isnan(dirty[i][130]).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_linear_autograd(cuda_lib, dt):
    t = dc.TORCH[dt]
    g = torch.Generator().manual_seed(2)
    shapes = ((2, 30, 64), (80, 64), (80,), (2, 30, 40))
    ref = [torch.randn(s, generator=g).to(t).double().requires_grad_() for s in shapes]
    leaves = [v.detach().to("cuda", t).requires_grad_() for v in ref]
    dy = torch.randn((2, 30, 40), generator=g).to(t)
    y = cuda_lib.sa_linear(leaves[0], leaves[1], leaves[2], "swiglu", leaves[3])
    y.backward(dy.cuda())
    z = ref[0] @ ref[1].T + ref[2]
    (torch.nn.functional.silu(z[..., :40]) * z[..., 40:] + ref[3]).backward(dy.double())
    for a, b in zip(leaves, ref):
        assert a.grad.dtype is t
        off = float((a.grad.cpu().double() - b.grad).norm() / b.grad.norm())
        assert off < (8e-3 if dt == "bf16" else 1e-5), off
    out = cuda_lib.sa_linear(leaves[0], leaves[1])
    dx, = torch.autograd.grad(out.float().square().sum(), leaves[0], create_graph=True)
    with pytest.raises(RuntimeError):
        dx.sum().backward()


def test_repeated_calls_give_the_same_bits(cuda_lib):
    for dt in ("bf16", "f32"):
        c = dc.linear_inputs(1500, 260, 200, "gelu", dt, 3)
        a = linear_call(cuda_lib, c, "gelu", dt)
        for _ in range(3):
            assert all(torch.equal(p, q) for p, q in zip(a, linear_call(cuda_lib, c, "gelu", dt)))
    c = dc.norm_inputs(3000, 200, 1, "f32", "bf16", "bf16")
    a = norm_call(cuda_lib, c, "f32", "bf16", "bf16")
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(a, norm_call(cuda_lib, c, "f32", "bf16", "bf16")))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(1, 70, 33), (4, 1030, 130), (5, 2052, 65), (16, 3001, 700), (16, 1024, 512), (3, 8, 4100)])
def test_linear_grads_of_few_rows(cuda_lib, shape, dt):
    """W read by columns and dW written row by row, over several strips and shares."""
    for act in ("none", "swiglu"):
        linear_check(cuda_lib, *shape, act, dt, seed=3)


def test_linear_grads_of_few_rows_unaligned(cuda_lib):
    """bf16 rows that TMA cannot read go the same way as fp32."""
    b = cuda_lib
    g = torch.Generator(device="cuda").manual_seed(6)
    wide = torch.randn((96, 525), generator=g, device="cuda").bfloat16()
    w, x = wide[:, 3:515], torch.randn((9, 512), generator=g, device="cuda").bfloat16()
    dy = torch.randn((9, 96), generator=g, device="cuda").bfloat16()
    got, want = b.sa_linear_bwd(dy, x, w), b.sa_linear_bwd(dy, x, w.contiguous())
    for p, q in zip(got, want):  # the same sums in another order
        assert float((p.float() - q.float()).norm()) <= 2e-3 * float(q.float().norm())
