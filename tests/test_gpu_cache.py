"""The 4-bit cache on the GPU: rows in and out, attention and the queries' gradient, against the
fp64 oracle at the sizes, masks, strides and streams where such kernels go wrong."""
import numpy as np
import pytest
import torch

import cache_cases as cc
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


def gpu(x, dtype=None):
    t = torch.as_tensor(x).to("cuda")
    return t if dtype is None else t.to(dtype)


# ------------------------------------------------------------------- rows

@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,page", [(64, 2, 64), (128, 3, 16), (96, 1, 32), (16, 5, 256), (48, 2, 128)])
def test_rows_read_back_as_the_stored_values(cuda_lib, dt, d, H, page):
    rng = np.random.default_rng(d + page)
    n = [0, 1, 33, page, 2 * page + 5]
    start = np.array([3, 0, page - 1, 0, 7], dtype=np.int32)
    cu = cc.offsets(n)
    N = int(cu[-1])
    std = np.exp(rng.uniform(-12, 9, (N, H, 1)))
    K, V = (cc.rounded(rng.standard_normal((N, H, d)) * std, dt) for _ in range(2))
    pages = [-(-(int(s) + m) // page) for s, m in zip(start, n)]
    table = np.full((5, max(pages)), -1, dtype=np.int32)
    order = rng.permutation(sum(pages) + 1)
    table[np.arange(max(pages))[None] < np.array(pages)[:, None]] = order[: sum(pages)]
    pool = cuda_lib.sa_cache_alloc(sum(pages) + 1, H, d, page)
    pool.fill_(0xAB)
    before = pool.clone()
    cuda_lib.sa_cache_write(pool, gpu(table), cc.to_gpu(K, dt), cc.to_gpu(V, dt), gpu(cu), start=gpu(start))
    for out in ("bf16", "f32"):
        k, v = cuda_lib.sa_cache_read(pool, gpu(table), gpu(cu), N, d, start=gpu(start), dtype=cc.TORCH[out])
        assert np.array_equal(k.double().cpu().numpy(), co.stored(K))
        assert np.array_equal(v.double().cpu().numpy(), co.stored(V))
    assert torch.equal(pool[order[-1]], before[order[-1]])  # nobody's page is untouched


def test_a_record_has_the_documented_bytes(cuda_lib):
    x = np.random.default_rng(3).standard_normal((16, 1, 48)).astype(np.float32)
    pool = cuda_lib.sa_cache_alloc(1, 1, 48, 16)
    table = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    cuda_lib.sa_cache_write(pool, table, gpu(x), gpu(-x), gpu(np.array([0, 16], np.int32)))
    got = pool.cpu().numpy()[0, 0]
    assert np.array_equal(got[0], co.record(x[:, 0]))
    assert np.array_equal(got[1], co.record(-x[:, 0]))


def test_values_at_the_format_s_edges(cuda_lib):
    rng = np.random.default_rng(4)
    rows = [np.zeros(16), np.full(16, np.inf), np.full(16, -np.inf), np.full(16, np.nan), np.full(16, 3.4e38),
            np.full(16, 1e-40), np.r_[np.nan, np.inf, np.arange(14)], np.full(16, -0.0)]
    for s in co.SCALES[::9]:  # every half of a step, and its neighbours
        mid = np.float32(s) * np.float32(7)
        half = (np.arange(15) / 2).astype(np.float32) * np.float32(s)
        for near in (half, np.nextafter(half, np.float32(1e30)), np.nextafter(half, np.float32(-1e30))):
            rows.append(np.r_[near, mid].astype(np.float64) * rng.choice([-1, 1], 16))
        edge = np.float32(s) * np.float32(7.5)  # where the next scale begins
        for e in (edge, np.nextafter(edge, np.float32(1e30)), np.nextafter(edge, np.float32(0))):
            rows.append(np.r_[np.full(15, s), e])
    x = np.stack(rows).astype(np.float32)[:, None]
    n = x.shape[0]
    pool = cuda_lib.sa_cache_alloc(-(-n // 16), 1, 16, 16)
    table = torch.arange(pool.shape[0], dtype=torch.int32, device="cuda")[None]
    cu = gpu(np.array([0, n], np.int32))
    cuda_lib.sa_cache_write(pool, table, gpu(x), gpu(x), cu)
    k, _ = cuda_lib.sa_cache_read(pool, table, cu, n, 16, dtype=torch.float32)
    assert np.array_equal(k.double().cpu().numpy(), co.stored(x.astype(np.float64)))


def test_sketches_and_strided_rows(cuda_lib):
    B, H, P, d, page = 3, 2, 40, 64, 32
    sketch = torch.randn((B, H, P, d), device="cuda")
    table = torch.arange(2 * B, dtype=torch.int32, device="cuda").flip(0).view(B, 2).contiguous()
    cu = gpu(cc.offsets([P] * B))
    pool = cuda_lib.sa_cache_alloc(2 * B, H, d, page)
    cuda_lib.sa_cache_write(pool, table, sketch, sketch)
    k, v = cuda_lib.sa_cache_read(pool, table, cu, B * P, d, dtype=torch.float32)
    want = co.stored(sketch.transpose(1, 2).reshape(B * P, H, d).double().cpu().numpy())
    assert np.array_equal(k.double().cpu().numpy(), want) and torch.equal(k, v)
    # K and V as two parts of one projection [N, 2, H, d + 16], heads reversed in memory order by a transpose
    both = torch.randn((H, B * P, 2, d + 16), device="cuda").bfloat16()
    K, V = (both[:, :, i, :d].transpose(0, 1) for i in range(2))
    cuda_lib.sa_cache_write(pool, table, K, V, cu)
    k, v = cuda_lib.sa_cache_read(pool, table, cu, B * P, d)
    assert np.array_equal(k.double().cpu().numpy(), co.stored(K.double().cpu().numpy()))
    assert np.array_equal(v.double().cpu().numpy(), co.stored(V.double().cpu().numpy()))


# --------------------------------------------------------------- attention

def run_both(lib, cache, n_q, G, dt, seed=0, scale=None, begin=None, end=None, std=1.0, q=None):
    """Forward and backward against the oracle; returns the GPU's (out, lse, dq)."""
    H, d = cache.H, cache.d
    T = int(np.sum(n_q))
    q = cc.queries(T, H * G, d, dt, seed, std) if q is None else q
    do = cc.queries(T, H * G, d, dt, seed + 77)
    scale = cc.default_scale(d) if scale is None else scale
    pool, table, lens = cache.tensors()
    kw = dict(scale=scale, kv_begin=None if begin is None else gpu(begin.astype(np.int32)),
              kv_end=None if end is None else gpu(end.astype(np.int32)))
    cu = gpu(cc.offsets(n_q))
    tq, tdo = cc.to_gpu(q, dt), cc.to_gpu(do, dt)
    out, lse = lib.sa_cache_attn_fwd(tq, cu, pool, table, lens, want_lse=True, **kw)
    dq = lib.sa_cache_attn_bwd(tq, cu, pool, table, lens, out, lse, tdo, **kw)
    torch.cuda.synchronize()
    for w in lib._stream_ws_cache.values():
        assert lib.sa_get_device_error(w) == 0
    r = cc.reference(cache, q, n_q, G, scale, begin, end, do, out.double().cpu().numpy(), lse.double().cpu().numpy())
    most = cc.limits(r, d, dt, max(1, max(cache.lens)))
    for name, got, m in zip(("out", "lse", "dq"), (out, lse, dq), most):
        cc.check(name, got, r[name], m)
    return out, lse, dq


LENS = [0, 1, 15, 63, 64, 65, 200, 129]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,G,page", [(64, 2, 1, 64), (128, 2, 1, 64), (128, 1, 16, 16), (64, 1, 5, 32),
                                        (96, 2, 2, 128), (32, 1, 3, 16), (80, 1, 1, 256), (16, 2, 4, 64)])
@pytest.mark.parametrize("R", [1, 9])
def test_ragged_batches(cuda_lib, dt, d, H, G, page, R):
    cache = cc.Cache(LENS, H, d, page, seed=d + G)
    n_q = [R, R, 0, R, 1, R + 2, R, 3] if R > 1 else [1] * 8
    run_both(cuda_lib, cache, n_q, G, dt, seed=R)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R", [1, 3, 40, 130, 300])
def test_many_queries(cuda_lib, dt, R):
    cache = cc.Cache([300, 77, 512], 2, 128, 64, seed=R)
    run_both(cuda_lib, cache, [R, max(1, R // 3), R], 2, dt, seed=R)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d,page,R", [(64, 16, 5), (128, 64, 20), (128, 128, 150), (64, 64, 150)])
def test_windows(cuda_lib, dt, d, page, R):
    cache = cc.Cache([0, 1, 190, 700, 333], 2, d, page, seed=9)
    n_q = [2, 3, R, R, 1]
    rng = np.random.default_rng(R)
    of = np.repeat(cache.lens, n_q)
    end = rng.integers(-2, of + 3)
    begin = np.maximum(-1, end - rng.integers(0, 200, of.size))
    begin[::7] = end[::7] + 1  # sees nothing
    run_both(cuda_lib, cache, n_q, 2, dt, begin=begin, end=end)
    run_both(cuda_lib, cache, n_q, 1, dt, begin=begin)
    run_both(cuda_lib, cache, n_q, 1, dt, end=end)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [-0.2, 0.0, 3.0])
@pytest.mark.parametrize("R", [2, 140])
def test_scales(cuda_lib, dt, scale, R):
    cache = cc.Cache([150, 260], 1, 64, 64, seed=3)
    run_both(cuda_lib, cache, [R, R], 1, dt, scale=scale)


@pytest.mark.parametrize("R", [1, 200])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_long_history_is_shared_out_and_joined(cuda_lib, dt, R):
    cache = cc.Cache([9001, 0, 4097], 1, 64, 64, seed=4)
    run_both(cuda_lib, cache, [R, 1, 1], 1, dt)


@pytest.mark.parametrize("d,R,L", [(128, 100, 300), (64, 100, 300), (64, 256, 130), (128, 140, 129)])
def test_many_segments_a_worker(cuda_lib, d, R, L):
    """More (user, head, row tile) segments than workers, of odd and even numbers of blocks, some empty."""
    lens = [(L * (3 + b % 5)) // 7 if b % 9 else 0 for b in range(200)]
    cache = cc.Cache(lens, 2, d, 64, seed=14)
    rng = np.random.default_rng(15)
    q = cc.queries(200 * R, 2, d, "bf16", 16)
    do = cc.queries(200 * R, 2, d, "bf16", 17)
    pool, table, tl = cache.tensors()
    cu = gpu(cc.offsets([R] * 200))
    tq = cc.to_gpu(q, "bf16")
    out, lse = cuda_lib.sa_cache_attn_fwd(tq, cu, pool, table, tl, want_lse=True)
    dq = cuda_lib.sa_cache_attn_bwd(tq, cu, pool, table, tl, out, lse, cc.to_gpu(do, "bf16"))
    torch.cuda.synchronize()
    for b in [int(x) for x in rng.choice(200, 12, replace=False)] + [0, 199]:
        rows = slice(b * R, (b + 1) * R)
        one = cc.Cache([0], 2, d, 64)
        one.lens, one.kv = [lens[b]], [[part[b]] for part in cache.kv]
        r = cc.reference(one, q[rows], [R], 1, cc.default_scale(d), dout=do[rows],
                         out=out[rows].double().cpu().numpy(), lse=lse[rows].double().cpu().numpy())
        for name, got, m in zip(("out", "lse", "dq"), (out, lse, dq), cc.limits(r, d, "bf16", max(1, lens[b]))):
            cc.check(name, got[rows], r[name], m)


@pytest.mark.parametrize("R", [1, 160])
def test_unwritten_and_hidden_positions_never_matter(cuda_lib, R):
    """Pages outside every query's window may be gone (-1) or hold anything."""
    cache = cc.Cache([500], 2, 128, 64, seed=6)
    begin, end = np.full(R, 200), np.full(R, 330)
    base = run_both(cuda_lib, cache, [R], 1, "bf16", begin=begin, end=end)
    cache.table[0, [0, 1, 2, 6, 7]] = -1
    gone = run_both(cuda_lib, cache, [R], 1, "bf16", begin=begin, end=end)
    rec = cache.pool[cache.table[0, 3]]  # positions 192..255: all before 200 overwritten
    rec[..., : 8 * 64] = 0xFF
    rec[..., 64 * 64: 64 * 64 + 8 * 8] = 0xFF
    dirty = run_both(cuda_lib, cache, [R], 1, "bf16", begin=begin, end=end)
    for a, b, c in zip(base, gone, dirty):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("R", [1, 160])
def test_one_query_s_nan_stays_its_own(cuda_lib, R):
    cache = cc.Cache([130], 1, 64, 64, seed=8)
    pool, table, lens = cache.tensors()
    cu = gpu(np.array([0, R + 1], np.int32))
    q = torch.randn((R + 1, 1, 64), device="cuda").bfloat16()
    ref = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens)
    q[R] = float("nan")
    got = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens)
    assert torch.equal(got[:R], ref[:R]) and torch.isnan(got[R]).all()


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("R", [3, 150])
def test_strided_queries_same_bits(cuda_lib, dt, R):
    cache = cc.Cache([300, 90], 2, 64, 32, seed=10)
    pool, table, lens = cache.tensors()
    cu = gpu(cc.offsets([R, R]))
    wide = torch.randn((4, 2 * R, 96), device="cuda").to(cc.TORCH[dt])
    q = wide[:, :, 16:80].transpose(0, 1)  # [T, 4, 64], head stride largest
    do = torch.randn((2 * R, 4, 64), device="cuda").to(cc.TORCH[dt])
    res = []
    for x in (q, q.contiguous()):
        out, lse = cuda_lib.sa_cache_attn_fwd(x, cu, pool, table, lens, want_lse=True)
        res.append((out, lse, cuda_lib.sa_cache_attn_bwd(x, cu, pool, table, lens, out, lse, do)))
    for a, b in zip(*res):
        assert torch.equal(a, b)


def test_autograd_against_the_call_and_differences(cuda_lib):
    cache = cc.Cache([70, 33], 1, 32, 16, seed=11)
    pool, table, lens = cache.tensors()
    cu = gpu(cc.offsets([2, 3]))
    q64 = cc.queries(5, 2, 32, "f32", 1)
    q = cc.to_gpu(q64, "f32").requires_grad_(True)
    g64 = cc.queries(5, 2, 32, "f32", 2)
    g = cc.to_gpu(g64, "f32")
    out = cuda_lib.sa_cache_attention(q, cu, pool, table, lens)
    out.backward(g)
    with torch.no_grad():
        o, l = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, want_lse=True)
        assert torch.equal(q.grad, cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, o, l, g))
    # differences of the oracle's fp64 forward along each coordinate: error h^2 / 6 f''' ~ 1e-9
    scale, h = 1.0 / np.sqrt(32.0), 1e-4
    got = q.grad.double().cpu().numpy()
    for t, hd, c in ((0, 0, 0), (1, 1, 31), (3, 0, 17), (4, 1, 5)):
        vals = []
        for s in (h, -h):
            x = q64.copy()
            x[t, hd, c] += s
            vals.append(np.sum(g64 * cc.reference(cache, x, [2, 3], 2, scale)["out"]))
        assert abs((vals[0] - vals[1]) / (2 * h) - got[t, hd, c]) < 2e-5


def test_same_bits_every_time_on_other_streams_and_in_a_graph(cuda_lib):
    cache = cc.Cache([3000, 10, 700], 2, 128, 64, seed=12)
    pool, table, lens = cache.tensors()
    for R in (1, 150):
        cu = gpu(cc.offsets([R, R, R]))
        q = torch.randn((3 * R, 4, 128), device="cuda").bfloat16()
        ref, lse = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, want_lse=True)
        dref = cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, ref, lse, q)
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        got = []
        for s in streams * 2:
            with torch.cuda.stream(s):
                o, l = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, want_lse=True)
                got.append((o, l, cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, o, l, q)))
        torch.cuda.synchronize()
        for o, l, dq in got:
            assert torch.equal(o, ref) and torch.equal(l, lse) and torch.equal(dq, dref)
        s = torch.cuda.Stream()
        with torch.cuda.stream(s):
            cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, ref, lse, q)  # the stream's workspace exists
            s.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                o, l = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, want_lse=True)
                dq = cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, o, l, q)
        for _ in range(2):
            o.zero_(), dq.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, ref) and torch.equal(l, lse) and torch.equal(dq, dref)


@pytest.mark.parametrize("R,G,lens", [(300, 1, [6000, 5100, 0, 2049]), (40, 16, [1024] * 6), (1, 1, [20000, 3, 900]),
                                      (100, 1, [700, 0, 130, 64] * 60)])
def test_many_calls_give_the_same_bits(cuda_lib, R, G, lens):
    """A wait on the wrong phase or a lost copy shows in one call of many."""
    cache = cc.Cache(lens, 1, 128, 64, seed=18)
    pool, table, tl = cache.tensors()
    B = len(lens)
    cu = gpu(cc.offsets([R] * B))
    q = torch.randn((B * R, G, 128), device="cuda").bfloat16()
    do = torch.randn((B * R, G, 128), device="cuda").bfloat16()
    ref, lse = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, tl, want_lse=True)
    dref = cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, tl, ref, lse, do)
    for _ in range(150):
        o, l = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, tl, want_lse=True)
        dq = cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, tl, ref, lse, do)
        assert torch.equal(o, ref) and torch.equal(l, lse) and torch.equal(dq, dref)
    for w in cuda_lib._stream_ws_cache.values():
        assert cuda_lib.sa_get_device_error(w) == 0


def test_offsets_past_32_bits(cuda_lib):
    """Pages beyond 4 GiB of the pool."""
    H, d, page = 8, 128, 256
    per = H * 2 * page * 72
    n_pages = (1 << 32) // per + 4
    pool = cuda_lib.sa_cache_alloc(n_pages, H, d, page)
    table = torch.tensor([[n_pages - 1, n_pages - 2]], dtype=torch.int32, device="cuda")
    K = torch.randn((300, H, d), device="cuda").bfloat16()
    cu = gpu(np.array([0, 300], np.int32))
    lens = gpu(np.array([300], np.int32))
    cuda_lib.sa_cache_write(pool, table, K, -K, cu)
    k, v = cuda_lib.sa_cache_read(pool, table, cu, 300, d)
    assert np.array_equal(k.double().cpu().numpy(), co.stored(K.double().cpu().numpy())) and torch.equal(k, -v)
    small = cuda_lib.sa_cache_alloc(2, H, d, page)
    t2 = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    cuda_lib.sa_cache_write(small, t2, K, -K, cu)
    for R in (1, 150):
        q = torch.randn((R, H, d), device="cuda").bfloat16()
        cq = gpu(np.array([0, R], np.int32))
        assert torch.equal(cuda_lib.sa_cache_attn_fwd(q, cq, pool, table, lens),
                           cuda_lib.sa_cache_attn_fwd(q, cq, small, t2, lens))


# ---------------------------------------------------------------- refusals

def test_device_detected_errors_are_reported_and_the_next_call_is_clean(cuda_lib):
    cache = cc.Cache([100, 60], 1, 64, 64, seed=13)
    pool, table, lens = cache.tensors()
    for R in (1, 150):
        q = torch.randn((2 * R, 1, 64), device="cuda").bfloat16()
        cu = gpu(cc.offsets([R, R]))
        ws = torch.empty(cuda_lib.sa_cache_attn_workspace_size(2, 2 * R, 1, 1, 64, 1, 128, False), dtype=torch.uint8,
                         device="cuda")

        def status(**kw):
            a = dict(cu_q=cu, block_table=table, cache_lens=lens)
            a.update(kw)
            cuda_lib.sa_cache_attn_fwd(q, a["cu_q"], pool, a["block_table"], a["cache_lens"], ws=ws)
            return cuda_lib.sa_get_device_error(ws)

        assert status() == 0
        assert status(cu_q=gpu(np.array([0, 2 * R + 1, 2 * R], np.int32))) == 6
        assert status(cu_q=gpu(np.array([0, R, 2 * R - 1], np.int32))) == 6
        assert status(cache_lens=gpu(np.array([100, 129], np.int32))) == 6
        assert status(cache_lens=gpu(np.array([-1, 60], np.int32))) == 6
        bad = table.clone()
        bad[0, 1] = pool.shape[0]
        assert status(block_table=bad) == 7
        bad[0, 1] = -1
        assert status(block_table=bad) == 7
        assert status() == 0
    K = torch.randn((160, 1, 64), device="cuda")
    w = torch.empty(256, dtype=torch.uint8, device="cuda")
    before = pool.clone()
    cuda_lib.sa_cache_write(pool, table, K, K, gpu(np.array([0, 170, 160], np.int32)), ws=w)
    assert cuda_lib.sa_get_device_error(w) == 6 and torch.equal(pool, before)
    cuda_lib.sa_cache_write(pool, table, K, K, gpu(np.array([0, 100, 160], np.int32)),
                            start=gpu(np.array([0, 69], np.int32)), ws=w)
    assert cuda_lib.sa_get_device_error(w) == 6
    bad = table.clone()
    bad[1, 0] = -1
    cuda_lib.sa_cache_write(pool, bad, K, K, gpu(np.array([0, 100, 160], np.int32)), ws=w)
    assert cuda_lib.sa_get_device_error(w) == 7
    cuda_lib.sa_cache_read(pool, table, gpu(np.array([0, 100, 160], np.int32)), 160, 64, ws=w)
    assert cuda_lib.sa_get_device_error(w) == 0


def test_the_binding_refuses(cuda_lib):
    cache = cc.Cache([64], 2, 64, 64)
    pool, table, lens = cache.tensors()
    cu = gpu(np.array([0, 3], np.int32))
    q = torch.randn((3, 2, 64), device="cuda").bfloat16()
    fwd = cuda_lib.sa_cache_attn_fwd
    with pytest.raises(ValueError):
        fwd(q.cpu(), cu, pool, table, lens)
    with pytest.raises(ValueError):
        fwd(q[..., :48], cu, pool, table, lens)  # not the pool's width
    with pytest.raises(ValueError):
        fwd(q[:, :1], cu, pool, table, lens)  # one query head over two cached heads
    with pytest.raises(ValueError):
        fwd(q, cu.long(), pool, table, lens)
    with pytest.raises(ValueError):
        fwd(q, cu, pool, table, lens.repeat(2))
    with pytest.raises(ValueError):
        fwd(q, cu, pool, table, lens, kv_end=lens)
    with pytest.raises(TypeError):
        fwd(q.half(), cu, pool, table, lens)
    with pytest.raises(cuda_lib.SketchError):
        fwd(q, cu, pool, table, lens, scale=float("inf"))
    with pytest.raises(cuda_lib.SketchError):
        fwd(q, cu, pool, table, lens, ws=torch.empty(256, dtype=torch.uint8, device="cuda"))
    out, lse = fwd(q, cu, pool, table, lens, want_lse=True)
    with pytest.raises(ValueError):
        cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, out, lse, out.float())
    with pytest.raises(ValueError):
        cuda_lib.sa_cache_write(pool, table, q, q.float(), cu)
    with pytest.raises(ValueError):
        cuda_lib.sa_cache_write(pool, table, q, q)  # packed rows need offsets
    with pytest.raises(cuda_lib.SketchError):
        cuda_lib.sa_cache_alloc(4, 1, 64, 48)


@pytest.mark.parametrize("R", [0, 5])
def test_no_queries_at_all(cuda_lib, R):
    cache = cc.Cache([64, 5], 2, 64, 64)
    pool, table, lens = cache.tensors()
    q = torch.randn((R, 2, 64), device="cuda").bfloat16()
    out, lse = cuda_lib.sa_cache_attn_fwd(q, gpu(np.array([0, 0, R], np.int32)), pool, table, lens, want_lse=True)
    assert out.shape == (R, 2, 64) and lse.shape == (R, 2) and torch.isfinite(out.float()).all()


def test_the_example_runs_the_operators_together(cuda_lib):
    from paper_2609_08443_gb300 import cached_targets

    res = cached_targets.run(lengths=(900, 300, 130), H=2, P=128, d=64, candidates=70)
    # a group's step is at most 1.125 / 7.5 of its largest value, its error uniform within half a step: under a
    # tenth of a row's norm in keys and in values together
    assert res["error"] < 0.2
    assert torch.isfinite(res["z"].float()).all() and res["dq"].abs().sum() > 0
    none = res["times"] == 0
    assert torch.isinf(res["lse"][none]).all() and not res["recent"][none].any()
    assert torch.isfinite(res["lse"][~none]).all()
    pages = res["recents"]
    held = [int(p) for p in pages.table.flatten() if p >= 0]
    assert len(held) == len(set(held)) and not set(held) & set(pages.free)
    pages.evict(0)
    assert pages.lens[0] == 0 and int(pages.table[0].max()) == -1
    with pytest.raises(RuntimeError):
        pages.grow(1, 10 ** 6)


@pytest.mark.parametrize("dt,R,L", [("bf16", 1, 70), ("f32", 2, 70), ("bf16", 160, 70), ("bf16", 1, 60000),
                                    ("bf16", 130, 60000)])
def test_a_nan_query_has_nan_for_its_sum_and_gradient(cuda_lib, dt, R, L):
    cache = cc.Cache([L], 1, 64, 64, seed=9)
    pool, table, lens = cache.tensors()
    cu = gpu(np.array([0, R + 1], np.int32))
    q = torch.randn((R + 1, 1, 64), device="cuda").to(cc.TORCH[dt])
    q[R, 0, 5] = float("nan")
    end = torch.full((R + 1,), L, dtype=torch.int32, device="cuda")
    for sees, value in ((True, float("nan")), (False, float("-inf"))):
        end[R] = L if sees else 0
        out, lse = cuda_lib.sa_cache_attn_fwd(q, cu, pool, table, lens, kv_end=end, want_lse=True)
        dq = cuda_lib.sa_cache_attn_bwd(q, cu, pool, table, lens, out, lse, torch.ones_like(q), kv_end=end)
        assert torch.isfinite(lse[:R]).all() and torch.isfinite(dq[:R]).all()
        if sees:
            assert torch.isnan(lse[R]).all() and torch.isnan(out[R]).all() and torch.isnan(dq[R]).all()
        else:
            assert lse[R].item() == value and not out[R].any() and not dq[R].any()


@pytest.mark.parametrize("d,bwd,rows", [(128, False, 32), (64, False, 40), (128, True, 40), (64, True, 56)])
def test_both_sides_of_the_choice_of_kernels(cuda_lib, d, bwd, rows):
    names = [cuda_lib.sa_cache_attn_kernel_name(3, 3 * r, 2, 2, d, 0.1, cuda_lib.SA_BF16, bwd) for r in (rows - 1, rows)]
    assert names[0].startswith("mma") and names[1].startswith("tc5")
    cache = cc.Cache([300, 77, 512], 2, d, 64, seed=rows)
    for r in (rows - 1, rows):
        run_both(cuda_lib, cache, [r, r, r], 1, "bf16", seed=r)
