"""Arguments that the binding refuses before any pointer reaches the library, without a GPU: device tensors
are played by host tensors that say they are on device 0."""
import pytest
import torch

from paper_2609_08443_gb300 import binding


class OnDevice(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0

    @classmethod
    def __torch_function__(cls, func, types, args=(), kwargs=None):
        with torch._C.DisableTorchFunctionSubclass():
            return func(*args, **(kwargs or {}))


def dev(*shape, dtype=torch.float32):
    return torch.zeros(shape, dtype=dtype).as_subclass(OnDevice)


class Library:
    """Takes every call: what gets here was not refused."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            if name == "sa_cache_attn_workspace_size":
                return 4096
            self.calls += 1
            return 0

        return call


@pytest.fixture
def lib(monkeypatch):
    library, empty = Library(), torch.empty
    monkeypatch.setattr(binding, "load", lambda: library)
    monkeypatch.setattr(binding, "_on", lambda index: binding._STAY)
    monkeypatch.setattr(binding, "_stream_handle", lambda index: 0)
    monkeypatch.setattr(binding, "_attn_workspace_size", lambda *a: 4096)
    monkeypatch.setattr(binding, "_stream_ws_cache", {})
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch, "empty", lambda *size, device=None, **kw: empty(*size, **kw).as_subclass(OnDevice))
    monkeypatch.setattr(torch, "empty_like", lambda t: empty(t.shape, dtype=t.dtype).as_subclass(OnDevice))
    yield library
    binding._own_ws.__dict__.clear()


def calls(**kw):
    """(the four calls, what each needs beside `kw`)."""
    pool, table = dev(4, 2, 2, 64 * 36, dtype=torch.uint8), dev(1, 2, dtype=torch.int32)
    q, two, one = dev(3, 2, 64), dev(2, dtype=torch.int32), dev(1, dtype=torch.int32)
    lse = dev(3, 2)

    def pick(**names):
        return {**names, **{k: v for k, v in kw.items() if k in names or k == "ws"}}

    return {
        "write": lambda: binding.sa_cache_write(**pick(pool=pool, block_table=table, K=q, V=q, cu_seqlens=two)),
        "read": lambda: binding.sa_cache_read(**pick(pool=pool, block_table=table, cu_seqlens=two, n_rows=3, d=64)),
        "fwd": lambda: binding.sa_cache_attn_fwd(**pick(q=q, cu_q=two, pool=pool, block_table=table, cache_lens=one)),
        "bwd": lambda: binding.sa_cache_attn_bwd(**pick(q=q, cu_q=two, pool=pool, block_table=table, cache_lens=one,
                                                        out=q, lse=lse, dout=q)),
    }


NAMES = ["write", "read", "fwd", "bwd"]


@pytest.mark.parametrize("name", NAMES)
def test_good_arguments_pass(lib, name):
    calls()[name]()
    calls(ws=dev(4096, dtype=torch.uint8))[name]()
    calls(ws=dev(4096))[name]()  # of any type, as bytes go a quarter of it
    assert lib.calls == 3


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("ws", [torch.zeros(4096, dtype=torch.uint8), dev(2, 4096, dtype=torch.uint8)[:, ::2],
                                dev(8192, dtype=torch.uint8)[::2], "ws"])
def test_a_workspace_that_is_no_device_memory_is_refused(lib, name, ws):
    """Its address and length go to the kernels as they are."""
    with pytest.raises(ValueError, match="ws"):
        calls(ws=ws)[name]()
    assert lib.calls == 0


@pytest.mark.parametrize("name,arg", [("read", "cu_seqlens"), ("fwd", "cu_q"), ("fwd", "cache_lens"), ("bwd", "cu_q"),
                                      ("bwd", "cache_lens")])
def test_offsets_and_lengths_are_required(lib, name, arg):
    with pytest.raises(ValueError, match=arg):
        calls(**{arg: None})[name]()
    assert lib.calls == 0
