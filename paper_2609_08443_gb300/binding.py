"""ctypes binding of libsa_sketch.so (argument marshalling only).

Every function here has the name of the C entry point it calls (see
``include/sa_sketch.h``, ``sa_cache.h`` and ``sa_dense.h``).  Torch supplies device memory and the current CUDA
stream; all arithmetic runs in the library's kernels.  If the library is not
built or cannot be loaded, every call raises: there is no CPU fallback.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import math
import os
import threading
from typing import Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "_lib", "libsa_sketch.so")

SA_F32, SA_BF16 = 0, 1
SA_KERNEL_FWD_MAIN, SA_KERNEL_BWD_MAIN, SA_KERNEL_AUX, SA_KERNEL_FWD_LSE, SA_KERNEL_BWD_DQ = 0, 1, 2, 3, 4
STATUS = {0: "SA_OK", 1: "SA_ERR_INVALID_ARG", 2: "SA_ERR_UNSUPPORTED", 3: "SA_ERR_WORKSPACE",
          4: "SA_ERR_CUDA", 5: "SA_ERR_TIMEOUT", 6: "SA_ERR_BAD_SEQLENS", 7: "SA_ERR_BAD_PAGE"}

_lib = None


class SketchError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {STATUS.get(status, status)} ({sa_status_string(status)})")


def load() -> ctypes.CDLL:
    """Load the CUDA library (raises if it is missing: no fallback exists)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    lib.sa_workspace_size.argtypes = [i32, i64, i32, i32, i32, i32, i32]
    lib.sa_workspace_size.restype = sz
    lib.sa_sketch_fwd.argtypes = [vp, vp, vp, i32, i64, vp, i32, i32, i32, f32, i32, vp, vp, vp, sz, vp]
    lib.sa_sketch_fwd.restype = i32
    lib.sa_sketch_bwd.argtypes = [vp, vp, vp, i32, i64, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp, vp,
                                  sz, vp]
    lib.sa_sketch_bwd.restype = i32
    lib.sa_get_device_error.argtypes = [vp, vp]
    lib.sa_get_device_error.restype = i32
    lib.sa_status_string.argtypes = [i32]
    lib.sa_status_string.restype = ctypes.c_char_p
    lib.sa_timing_enable.argtypes = [i32]
    lib.sa_timing_enable.restype = i32
    lib.sa_timing_read.argtypes = [i32, ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int64)]
    lib.sa_timing_read.restype = i32
    lib.sa_launch_count.argtypes = []
    lib.sa_launch_count.restype = ctypes.c_uint64
    lib.sa_main_kernel_name.argtypes = [i32, i32, i32, i32]
    lib.sa_main_kernel_name.restype = ctypes.c_char_p
    lib.sa_select_path.argtypes = [i32]
    lib.sa_select_path.restype = i32
    lib.sa_sketch_fwd_per_user.argtypes = lib.sa_sketch_fwd.argtypes
    lib.sa_sketch_fwd_per_user.restype = i32
    lib.sa_sketch_bwd_per_user.argtypes = lib.sa_sketch_bwd.argtypes
    lib.sa_sketch_bwd_per_user.restype = i32
    lib.sa_workspace_size_x.argtypes = [i32, i64, i32, i32, i32, i32, i32]
    lib.sa_workspace_size_x.restype = sz
    lib.sa_sketch_fwd_x.argtypes = [vp, vp, i32, i64, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, sz, vp]
    lib.sa_sketch_fwd_x.restype = i32
    lib.sa_sketch_bwd_x.argtypes = [vp, vp, i32, i64, vp, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp, vp,
                                    sz, vp]
    lib.sa_sketch_bwd_x.restype = i32
    lib.sa_sketch_fwd_noalloc.argtypes = [vp, vp, vp, i32, i64, vp, i32, i32, i32, f32, i32, vp, vp, vp]
    lib.sa_sketch_fwd_noalloc.restype = i32
    lib.sa_noalloc_scratch_bytes.argtypes = []
    lib.sa_noalloc_scratch_bytes.restype = sz
    lib.sa_noalloc_get_device_error.argtypes = [vp]
    lib.sa_noalloc_get_device_error.restype = i32
    lib.sa_set_wait_limit_ns.argtypes = [ctypes.c_uint64]
    lib.sa_set_wait_limit_ns.restype = i32
    lib.sa_workspace_size_tokenwise.argtypes = [i32, i64, i32, i32, i32, i32, i32]
    lib.sa_workspace_size_tokenwise.restype = sz
    lib.sa_sketch_fwd_tokenwise.argtypes = lib.sa_sketch_fwd.argtypes
    lib.sa_sketch_fwd_tokenwise.restype = i32
    lib.sa_sketch_bwd_tokenwise.argtypes = [vp, vp, vp, i32, i64, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp,
                                            vp, vp, sz, vp]
    lib.sa_sketch_bwd_tokenwise.restype = i32
    lib.sa_step_host_workspace_size.argtypes = [vp, i32, i32, i32, i32, i32, i64]
    lib.sa_step_host_workspace_size.restype = sz
    lib.sa_sketch_step_host.argtypes = [vp, vp, vp, i32, i64, vp, i32, i32, i32, f32, i32, vp, vp, vp, vp, vp, i64,
                                        vp, sz, vp]
    lib.sa_sketch_step_host.restype = i32
    lib.sa_plan_chunks_host.argtypes = [vp, i32, i64, vp, vp]
    lib.sa_plan_chunks_host.restype = i32
    lib.sa_plan_host.argtypes = [vp, i32, i32, i32, i32, vp]
    lib.sa_plan_host.restype = i32
    lib.sa_walk_host.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, ctypes.c_int64]
    lib.sa_walk_host.restype = i32
    lib.sa_cache_page_bytes.argtypes = [i32, i32, i32]
    lib.sa_cache_page_bytes.restype = sz
    lib.sa_cache_write.argtypes = [vp, vp, i64, i64, i64, vp, i32, i64, vp, i32, i32, i32, vp, i64, i32, vp, i32, vp,
                                   sz, vp]
    lib.sa_cache_write.restype = i32
    lib.sa_cache_read.argtypes = [vp, i64, i32, vp, i32, vp, i32, i64, vp, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.sa_cache_read.restype = i32
    lib.sa_cache_attn_workspace_size.argtypes = [i32, i64, i32, i32, i32, i32, i64, i32]
    lib.sa_cache_attn_workspace_size.restype = sz
    attn = [vp, i64, i64, vp, i32, i64, i32, vp, i64, i32, vp, i32, vp, i32, i32, vp, vp, f32, i32]
    lib.sa_cache_attn_fwd.argtypes = attn + [vp, vp, vp, sz, vp]
    lib.sa_cache_attn_fwd.restype = i32
    lib.sa_cache_attn_bwd.argtypes = attn + [vp, vp, vp, vp, vp, sz, vp]
    lib.sa_cache_attn_bwd.restype = i32
    lib.sa_cache_attn_kernel_name.argtypes = [i32, i64, i32, i32, i32, f32, i32, i32]
    lib.sa_cache_attn_kernel_name.restype = ctypes.c_char_p
    lib.sa_layer_norm_fwd.argtypes = [vp, i64, i32, vp, i64, i32, vp, vp, i32, i64, i32, f32, vp, i32, vp, vp]
    lib.sa_layer_norm_fwd.restype = i32
    lib.sa_layer_norm_workspace_size.argtypes = [i64, i32]
    lib.sa_layer_norm_workspace_size.restype = sz
    lib.sa_layer_norm_bwd.argtypes = [vp, i64, i32, vp, i64, i32, vp, i64, i32, vp, i32, vp, i64, i32, vp, vp, vp, vp,
                                      vp, sz, vp]
    lib.sa_layer_norm_bwd.restype = i32
    lib.sa_linear_workspace_size.argtypes = [i64, i32, i32, i32, i32, i32, i32]
    lib.sa_linear_workspace_size.restype = sz
    lib.sa_linear_fwd.argtypes = [vp, i64, vp, i64, vp, vp, i64, i64, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.sa_linear_fwd.restype = i32
    lib.sa_linear_bwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, i32, i32, vp, vp, vp, vp, sz, vp]
    lib.sa_linear_bwd.restype = i32
    lib.sa_linear_kernel_name.argtypes = [i64, i32, i32, i32, i32, i32]
    lib.sa_linear_kernel_name.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return SA_BF16
    if t.dtype == torch.float32:
        return SA_F32
    raise TypeError(f"unsupported dtype {t.dtype} (bf16 or fp32)")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(torch.cuda.current_stream(device).cuda_stream)


def _check(st: int, where: str):
    if st != 0:
        raise SketchError(st, where)


def _validate(K, V, cu, Q):
    for name, t in (("K", K), ("V", V), ("Q", Q), ("cu_seqlens", cu)):
        if not t.is_cuda:
            raise ValueError(f"{name} must be a CUDA tensor")
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
    # Q [H,P,d] (prototypes shared by all users) or [B,H,P,d] (per-user queries, Sec. 3.3)
    shared_ok = Q.dim() == 3 and Q.shape[0] == K.shape[1] and Q.shape[2] == K.shape[2]
    per_user_ok = (Q.dim() == 4 and Q.shape[0] == cu.numel() - 1 and Q.shape[1] == K.shape[1]
                   and Q.shape[3] == K.shape[2])
    if K.dim() != 3 or V.shape != K.shape or not (shared_ok or per_user_ok):
        raise ValueError(f"shapes K{tuple(K.shape)} V{tuple(V.shape)} Q{tuple(Q.shape)}: want K,V [N,H,d], "
                         "Q [H,P,d] or [B,H,P,d]")
    if K.dtype != V.dtype or K.dtype != Q.dtype:
        raise ValueError("K, V and Q must share one dtype")
    if cu.dtype != torch.int32 or cu.dim() != 1 or cu.numel() < 2:
        raise ValueError("cu_seqlens must be int32 [B+1]")


# ------------------------------------------------------------- C entry points

def sa_workspace_size(B: int, N: int, H: int, P: int, d: int, dt: int, bwd: bool) -> int:
    return int(load().sa_workspace_size(B, N, H, P, d, dt, int(bool(bwd))))


def sa_status_string(status: int) -> str:
    return load().sa_status_string(status).decode()


def sa_main_kernel_name(P: int, d: int, dt: int, bwd: bool) -> str:
    return load().sa_main_kernel_name(P, d, dt, int(bool(bwd))).decode()


def sa_launch_count() -> int:
    return int(load().sa_launch_count())


def sa_select_path(path: int) -> None:
    """0: tensor-core kernels where supported (default); 1: CUDA cores only;
    2: tensor cores with the lse pass + prototype slices for P = 512."""
    _check(load().sa_select_path(int(path)), "sa_select_path")


def sa_timing_enable(on: bool) -> None:
    _check(load().sa_timing_enable(int(bool(on))), "sa_timing_enable")


def sa_timing_read(kernel_class: int) -> Tuple[float, int]:
    ms, n = ctypes.c_double(), ctypes.c_int64()
    _check(load().sa_timing_read(kernel_class, ctypes.byref(ms), ctypes.byref(n)), "sa_timing_read")
    return ms.value, n.value


def sa_get_device_error(workspace: torch.Tensor) -> int:
    return int(load().sa_get_device_error(_ptr(workspace), _stream(workspace.device)))


_ws_cache = {}


def workspace(nbytes: int, device) -> torch.Tensor:
    """A cached uint8 device buffer of at least ``nbytes`` (allocated by torch)."""
    dev = torch.device(device)
    key = (dev.type, dev.index if dev.index is not None else torch.cuda.current_device())
    buf = _ws_cache.get(key)
    if buf is None or buf.numel() < nbytes:
        buf = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=dev)
        _ws_cache[key] = buf
    return buf


def sa_sketch_fwd(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                  scale: Optional[float] = None, want_lse: bool = False,
                  out: Optional[torch.Tensor] = None, lse_out: Optional[torch.Tensor] = None,
                  ws: Optional[torch.Tensor] = None):
    """sketch [B,H,P,d] fp32 (and lse [N,H] fp32 when ``want_lse``).  Q is
    [H,P,d] (C: sa_sketch_fwd) or per user [B,H,P,d] (C: sa_sketch_fwd_per_user)."""
    lib = load()
    _validate(K, V, cu_seqlens, Q)
    N, H, d = K.shape
    P = Q.shape[-2]
    entry = lib.sa_sketch_fwd_per_user if Q.dim() == 4 else lib.sa_sketch_fwd
    B = cu_seqlens.numel() - 1
    dt = _dt(K)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    sketch = out if out is not None else torch.empty((B, H, P, d), dtype=torch.float32, device=K.device)
    lse = lse_out if lse_out is not None else (
        torch.empty((N, H), dtype=torch.float32, device=K.device) if want_lse else None)
    need = lib.sa_workspace_size(B, N, H, P, d, dt, 0)
    if need == 0:
        raise SketchError(2, "sa_workspace_size")
    w = ws if ws is not None else workspace(need, K.device)
    st = entry(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale, dt,
               _ptr(sketch), _ptr(lse), _ptr(w), w.numel(), _stream(K.device))
    _check(st, "sa_sketch_fwd_per_user" if Q.dim() == 4 else "sa_sketch_fwd")
    return (sketch, lse) if want_lse or lse_out is not None else sketch


def sa_sketch_bwd(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                  dsketch: torch.Tensor, scale: Optional[float] = None,
                  lse: Optional[torch.Tensor] = None, outs=None, ws: Optional[torch.Tensor] = None):
    """(dK, dV, dQ): dK, dV like K; dQ fp32 shaped like Q ([H,P,d] summed over
    users, or [B,H,P,d] per user: C sa_sketch_bwd / sa_sketch_bwd_per_user)."""
    lib = load()
    _validate(K, V, cu_seqlens, Q)
    N, H, d = K.shape
    P = Q.shape[-2]
    entry = lib.sa_sketch_bwd_per_user if Q.dim() == 4 else lib.sa_sketch_bwd
    B = cu_seqlens.numel() - 1
    if dsketch.shape != (B, H, P, d) or dsketch.dtype != torch.float32 or not dsketch.is_contiguous():
        raise ValueError("dsketch must be contiguous fp32 [B,H,P,d]")
    if lse is not None and (lse.shape != (N, H) or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse must be contiguous fp32 [N,H]")
    dt = _dt(K)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    if outs is None:
        dK, dV = torch.empty_like(K), torch.empty_like(V)
        dQ = torch.empty(tuple(Q.shape), dtype=torch.float32, device=K.device)
    else:
        dK, dV, dQ = outs
    need = lib.sa_workspace_size(B, N, H, P, d, dt, 1)
    if need == 0:
        raise SketchError(2, "sa_workspace_size")
    w = ws if ws is not None else workspace(need, K.device)
    st = entry(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale, dt,
               _ptr(dsketch), _ptr(lse), _ptr(dK), _ptr(dV), _ptr(dQ), _ptr(w), w.numel(), _stream(K.device))
    _check(st, "sa_sketch_bwd_per_user" if Q.dim() == 4 else "sa_sketch_bwd")
    return dK, dV, dQ


def sa_sketch_fwd_per_user(K, V, cu_seqlens, Q, scale=None, **kw):
    """Forward with per-user queries Q [B,H,P,d] (stacked refinement, Sec. 3.3)."""
    if Q.dim() != 4:
        raise ValueError("per-user queries are [B,H,P,d]")
    return sa_sketch_fwd(K, V, cu_seqlens, Q, scale, **kw)


def sa_sketch_bwd_per_user(K, V, cu_seqlens, Q, dsketch, scale=None, **kw):
    """Backward with per-user queries: dQ [B,H,P,d], each user's own gradient."""
    if Q.dim() != 4:
        raise ValueError("per-user queries are [B,H,P,d]")
    return sa_sketch_bwd(K, V, cu_seqlens, Q, dsketch, scale, **kw)


def sa_sketch_fwd_noalloc(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                          scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                          lse_out: Optional[torch.Tensor] = None):
    """Forward without a workspace: for callers that may not allocate device
    memory when they run this (the library's fixed scratch array is used; see
    include/sa_sketch.h).  ``out`` and ``lse_out`` are the caller's buffers;
    when they are not given they are created here, before the call."""
    lib = load()
    _validate(K, V, cu_seqlens, Q)
    N, H, d = K.shape
    if Q.dim() != 3:
        raise ValueError("sa_sketch_fwd_noalloc takes shared prototypes Q [H,P,d]")
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    sketch = out if out is not None else torch.empty((B, H, P, d), dtype=torch.float32, device=K.device)
    # the library uses the fixed array of the CURRENT device: make K's device current
    with torch.cuda.device(K.device):
        st = lib.sa_sketch_fwd_noalloc(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale,
                                       _dt(K), _ptr(sketch), _ptr(lse_out), _stream(K.device))
    _check(st, "sa_sketch_fwd_noalloc")
    return sketch


def sa_noalloc_get_device_error(device=None) -> int:
    """Device-detected status of the last sa_sketch_fwd_noalloc call on
    ``device`` (synchronises its current stream)."""
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    with torch.cuda.device(device):
        return int(load().sa_noalloc_get_device_error(_stream(device)))


def sa_set_wait_limit_ns(ns: int) -> None:
    """Limit of the kernels' bounded pipeline waits for later calls (0 = the
    default 2 s); a test hook for the timeout path."""
    _check(load().sa_set_wait_limit_ns(int(ns)), "sa_set_wait_limit_ns")


def _validate_x(X, cu, Q, Wk):
    for name, t in (("X", X), ("Q", Q), ("Wk", Wk), ("cu_seqlens", cu)):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CUDA tensor")
    N, H, d = X.shape
    if Q.dim() != 3 or Q.shape[0] != H or Q.shape[2] != d or tuple(Wk.shape) != (H, d, d):
        raise ValueError(f"shapes X{tuple(X.shape)} Q{tuple(Q.shape)} Wk{tuple(Wk.shape)}: "
                         "want X [N,H,d], Q [H,P,d], Wk [H,d,d]")
    if X.dtype != Q.dtype or X.dtype != Wk.dtype:
        raise ValueError("X, Q and Wk must share one dtype")
    if cu.dtype != torch.int32 or cu.dim() != 1 or cu.numel() < 2:
        raise ValueError("cu_seqlens must be int32 [B+1]")


def sa_sketch_fwd_x(X: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor, Wk: torch.Tensor,
                    scale: Optional[float] = None, want_lse: bool = False, ws: Optional[torch.Tensor] = None):
    """Sketch with keys X Wk[h] and values X (Sec. 3.1): [B,H,P,d] fp32 (and lse)."""
    lib = load()
    _validate_x(X, cu_seqlens, Q, Wk)
    N, H, d = X.shape
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    dt = _dt(X)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    sketch = torch.empty((B, H, P, d), dtype=torch.float32, device=X.device)
    lse = torch.empty((N, H), dtype=torch.float32, device=X.device) if want_lse else None
    need = lib.sa_workspace_size_x(B, N, H, P, d, dt, 0)
    if need == 0:
        raise SketchError(2, "sa_workspace_size_x")
    w = ws if ws is not None else workspace(need, X.device)
    st = lib.sa_sketch_fwd_x(_ptr(X), _ptr(cu_seqlens), B, N, _ptr(Q), _ptr(Wk), H, P, d, scale, dt,
                             _ptr(sketch), _ptr(lse), _ptr(w), w.numel(), _stream(X.device))
    _check(st, "sa_sketch_fwd_x")
    return (sketch, lse) if want_lse else sketch


def sa_sketch_bwd_x(X: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor, Wk: torch.Tensor,
                    dsketch: torch.Tensor, scale: Optional[float] = None, lse: Optional[torch.Tensor] = None,
                    ws: Optional[torch.Tensor] = None):
    """(dX like X, dQ [H,P,d] fp32, dWk [H,d,d] fp32) for ``sa_sketch_fwd_x``."""
    lib = load()
    _validate_x(X, cu_seqlens, Q, Wk)
    N, H, d = X.shape
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    if dsketch.shape != (B, H, P, d) or dsketch.dtype != torch.float32 or not dsketch.is_contiguous():
        raise ValueError("dsketch must be contiguous fp32 [B,H,P,d]")
    dt = _dt(X)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dX = torch.empty_like(X)
    dQ = torch.empty((H, P, d), dtype=torch.float32, device=X.device)
    dWk = torch.empty((H, d, d), dtype=torch.float32, device=X.device)
    need = lib.sa_workspace_size_x(B, N, H, P, d, dt, 1)
    if need == 0:
        raise SketchError(2, "sa_workspace_size_x")
    w = ws if ws is not None else workspace(need, X.device)
    st = lib.sa_sketch_bwd_x(_ptr(X), _ptr(cu_seqlens), B, N, _ptr(Q), _ptr(Wk), H, P, d, scale, dt,
                             _ptr(dsketch), _ptr(lse), _ptr(dX), _ptr(dQ), _ptr(dWk), _ptr(w), w.numel(),
                             _stream(X.device))
    _check(st, "sa_sketch_bwd_x")
    return dX, dQ, dWk


def sa_sketch_fwd_tokenwise(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                            scale: Optional[float] = None, want_lse: bool = False,
                            ws: Optional[torch.Tensor] = None):
    """Token-wise normalisation (Sec. 5.1, App. C): sketch [B,H,P,d] fp32 with
    weights softmax over each user's tokens per prototype (and lse_tok [B,H,P])."""
    lib = load()
    _validate(K, V, cu_seqlens, Q)
    if Q.dim() != 3:
        raise ValueError("the token-wise variant takes shared prototypes Q [H,P,d]")
    N, H, d = K.shape
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    dt = _dt(K)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    sketch = torch.empty((B, H, P, d), dtype=torch.float32, device=K.device)
    lse = torch.empty((B, H, P), dtype=torch.float32, device=K.device) if want_lse else None
    need = lib.sa_workspace_size_tokenwise(B, N, H, P, d, dt, 0)
    if need == 0:
        raise SketchError(2, "sa_workspace_size_tokenwise")
    w = ws if ws is not None else workspace(need, K.device)
    st = lib.sa_sketch_fwd_tokenwise(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale, dt,
                                     _ptr(sketch), _ptr(lse), _ptr(w), w.numel(), _stream(K.device))
    _check(st, "sa_sketch_fwd_tokenwise")
    return (sketch, lse) if want_lse else sketch


def sa_sketch_bwd_tokenwise(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                            dsketch: torch.Tensor, scale: Optional[float] = None,
                            sketch: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                            ws: Optional[torch.Tensor] = None):
    """(dK, dV, dQ [H,P,d] fp32) of ``sa_sketch_fwd_tokenwise``; ``sketch`` and
    ``lse`` are the forward's outputs (recomputed when either is missing)."""
    lib = load()
    _validate(K, V, cu_seqlens, Q)
    if Q.dim() != 3:
        raise ValueError("the token-wise variant takes shared prototypes Q [H,P,d]")
    N, H, d = K.shape
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    for name, t, shape in (("dsketch", dsketch, (B, H, P, d)), ("sketch", sketch, (B, H, P, d)),
                           ("lse", lse, (B, H, P))):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.float32 or not t.is_contiguous()):
            raise ValueError(f"{name} must be contiguous fp32 {list(shape)}")
    dt = _dt(K)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dK, dV = torch.empty_like(K), torch.empty_like(V)
    dQ = torch.empty((H, P, d), dtype=torch.float32, device=K.device)
    need = lib.sa_workspace_size_tokenwise(B, N, H, P, d, dt, 1)
    if need == 0:
        raise SketchError(2, "sa_workspace_size_tokenwise")
    w = ws if ws is not None else workspace(need, K.device)
    st = lib.sa_sketch_bwd_tokenwise(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale, dt,
                                     _ptr(sketch), _ptr(lse), _ptr(dsketch), _ptr(dK), _ptr(dV), _ptr(dQ),
                                     _ptr(w), w.numel(), _stream(K.device))
    _check(st, "sa_sketch_bwd_tokenwise")
    return dK, dV, dQ


def sa_sketch_step_host(K: torch.Tensor, V: torch.Tensor, cu_seqlens: torch.Tensor, Q: torch.Tensor,
                        dsketch: torch.Tensor, scale: Optional[float] = None, chunk_tokens: int = 0,
                        outs=None, device=None, ws: Optional[torch.Tensor] = None):
    """Forward + backward of a batch held in host memory (C: sa_sketch_step_host):
    K, V [N,H,d], cu_seqlens [B+1] int32, Q [H,P,d], dsketch [B,H,P,d] fp32, all
    CPU tensors (page-locked for overlapped copies).  Returns CPU tensors
    (sketch, dK, dV, dQ), written once the current stream of ``device`` is
    synchronised (this function synchronises it before returning)."""
    lib = load()
    for name, t in (("K", K), ("V", V), ("Q", Q), ("cu_seqlens", cu_seqlens), ("dsketch", dsketch)):
        if t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous CPU tensor")
    N, H, d = K.shape
    P = Q.shape[1]
    B = cu_seqlens.numel() - 1
    if cu_seqlens.dtype != torch.int32 or V.shape != K.shape or tuple(Q.shape) != (H, P, d) or \
            tuple(dsketch.shape) != (B, H, P, d) or dsketch.dtype != torch.float32:
        raise ValueError("shapes: K,V [N,H,d], Q [H,P,d], cu_seqlens int32 [B+1], dsketch fp32 [B,H,P,d]")
    dt = _dt(K)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    if outs is None:
        pin = K.is_pinned()
        outs = (torch.empty((B, H, P, d), dtype=torch.float32, pin_memory=pin),
                torch.empty_like(K, pin_memory=pin), torch.empty_like(V, pin_memory=pin),
                torch.empty((H, P, d), dtype=torch.float32, pin_memory=pin))
    sketch, dK, dV, dQ = outs
    need = lib.sa_step_host_workspace_size(_ptr(cu_seqlens), B, H, P, d, dt, int(chunk_tokens))
    if need == 0:
        raise SketchError(2, "sa_step_host_workspace_size")
    w = ws if ws is not None else workspace(need, dev)
    st = lib.sa_sketch_step_host(_ptr(K), _ptr(V), _ptr(cu_seqlens), B, N, _ptr(Q), H, P, d, scale, dt,
                                 _ptr(dsketch), _ptr(sketch), _ptr(dK), _ptr(dV), _ptr(dQ), int(chunk_tokens),
                                 _ptr(w), w.numel(), _stream(dev))
    _check(st, "sa_sketch_step_host")
    torch.cuda.current_stream(dev).synchronize()
    return sketch, dK, dV, dQ


def sa_plan_chunks_host(cu_seqlens_host, chunk_tokens: int = 0):
    """Chunk boundaries (user indices) sa_sketch_step_host uses (pure C; no GPU)."""
    import numpy as np

    cu = np.ascontiguousarray(cu_seqlens_host, dtype=np.int32)
    begin = np.zeros(cu.size, dtype=np.int32)
    n = ctypes.c_int()
    st = load().sa_plan_chunks_host(cu.ctypes.data, cu.size - 1, int(chunk_tokens), begin.ctypes.data,
                                    ctypes.byref(n))
    _check(st, "sa_plan_chunks_host")
    return begin[: n.value + 1]


def sa_noalloc_scratch_bytes() -> int:
    return int(load().sa_noalloc_scratch_bytes())


def sa_plan_host(cu_seqlens_host, H: int, tile: int, n_workers: int):
    """Host copy of the tiling every call applies (pure C; no GPU)."""
    import numpy as np

    cu = np.ascontiguousarray(cu_seqlens_host, dtype=np.int32)
    begin = np.zeros(n_workers + 1, dtype=np.int64)
    st = load().sa_plan_host(cu.ctypes.data, cu.size - 1, H, tile, n_workers, begin.ctypes.data)
    _check(st, "sa_plan_host")
    return begin


# ------------------------------------------------------------------ autograd

class SketchAttention(torch.autograd.Function):
    """sketch = softmax_proto(scale Q K^T) V per user and head (Sec. 3.1)."""

    @staticmethod
    def forward(ctx, K, V, cu_seqlens, Q, scale):
        sketch, lse = sa_sketch_fwd(K, V, cu_seqlens, Q, scale, want_lse=True)
        ctx.save_for_backward(K, V, cu_seqlens, Q, lse)
        ctx.scale = scale
        return sketch

    @staticmethod
    def backward(ctx, dsketch):
        K, V, cu, Q, lse = ctx.saved_tensors
        dK, dV, dQ = sa_sketch_bwd(K, V, cu, Q, dsketch.contiguous(), ctx.scale, lse=lse)
        return dK, dV, None, dQ.to(Q.dtype), None


def sa_walk_host(cu_seqlens_host, H: int, tile: int, n_workers: int):
    """(user, head, tok0, ntok) of every tile in the order the kernels' workers
    walk them (C: sa_walk_host; pure C, no GPU)."""
    import numpy as np

    cu = np.ascontiguousarray(cu_seqlens_host, dtype=np.int32)
    L = np.diff(cu.astype(np.int64))
    total = int(np.sum((np.maximum(L, 0) + tile - 1) // tile)) * H
    out = (np.zeros(max(total, 1), np.int32), np.zeros(max(total, 1), np.int32), np.zeros(max(total, 1), np.int64),
           np.zeros(max(total, 1), np.int32))
    st = load().sa_walk_host(cu.ctypes.data, cu.size - 1, H, tile, n_workers, *(o.ctypes.data for o in out),
                             max(total, 1))
    _check(st, "sa_walk_host")
    return tuple(o[:total] for o in out)


def sa_sketch(K, V, cu_seqlens, Q, scale: Optional[float] = None):
    """Differentiable sketch [B,H,P,d] (fp32) of packed ragged histories."""
    scale = 1.0 / math.sqrt(K.shape[-1]) if scale is None else float(scale)
    return SketchAttention.apply(K, V, cu_seqlens, Q, scale)


# ------------------------------------------------------- the 4-bit cache
# (include/sa_cache.h).  `pool` is uint8 [n_pages, H, 2, page * (d/2 + d/16)] and
# `block_table` int32 [B, max_pages]; the page size follows from the pool's shape
# and the width d of the rows.

# A thread's workspaces, one for each of the streams that it used last, and, for their status,
# the workspaces of each stream's latest call from any thread.
_own_ws = threading.local()
_stream_ws_cache = {}
_STREAMS_KEPT = 8
_ws_lock = threading.Lock()


# These calls answer single tokens, so their checks avoid what costs a microsecond in
# Python: device and stream objects, and properties read twice.

def _addr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _on(index: int):
    """Makes device ``index`` current for a call (nothing to do, and no cost, where it is)."""
    return _STAY if torch.cuda.current_device() == index else torch.cuda.device(index)


_STAY = contextlib.nullcontext()


def _stream_handle(index: int) -> int:
    """The current stream of a device, without building its Python object where torch lets us."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return raw(index) if raw is not None else torch.cuda.current_stream(index).cuda_stream


def _keep(kept: dict, key, buf: torch.Tensor) -> None:
    with _ws_lock:
        kept.pop(key, None)
        while len(kept) >= _STREAMS_KEPT:
            del kept[next(iter(kept))]
        kept[key] = buf


def _stream_workspace(nbytes: int, index: int, stream: int, kept: threading.local = _own_ws) -> torch.Tensor:
    """Memory for one call on the current stream.  A thread's calls on a stream come one after the other and
    share one buffer.  Two threads' calls may interleave, a call being two launches, and have their own; so has
    a captured call, whose graph may run at any time and on any stream (its pool keeps what the call took)."""
    key = (index, stream)
    if torch.cuda.is_current_stream_capturing():
        buf = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", index))
    else:
        own = kept.__dict__
        buf = own.get(key)
        if buf is None or buf.numel() < nbytes:
            buf = torch.empty(nbytes, dtype=torch.uint8, device=torch.device("cuda", index))
            _keep(own, key, buf)
    return buf


def _note_call(buf: torch.Tensor, index: int, stream: int, kept: dict = _stream_ws_cache) -> None:
    """``buf`` holds the status of the stream's latest call."""
    if kept.get((index, stream)) is not buf:
        _keep(kept, (index, stream), buf)


def sa_cache_get_device_error(device=None) -> int:
    """Status of the latest sa_cache_* call on the current stream (from any thread) that was given no ``ws``:
    0, or what the device found (SA_ERR_TIMEOUT, SA_ERR_BAD_SEQLENS, SA_ERR_BAD_PAGE).  Waits for the stream.
    A captured call's status is that of its graph's last replay: wait for the stream that ran it first."""
    return _kept_status(device, _stream_ws_cache)


def _kept_status(device, kept: dict) -> int:
    index = torch.device("cuda" if device is None else device).index
    index = torch.cuda.current_device() if index is None else index
    with _on(index):
        buf = kept.get((index, _stream_handle(index)))
        return 0 if buf is None else sa_get_device_error(buf)


def sa_cache_page_bytes(H: int, d: int, page: int) -> int:
    """Bytes of one page of ``page`` tokens (0 for unsupported sizes)."""
    return int(load().sa_cache_page_bytes(H, d, page))


def sa_cache_alloc(n_pages: int, H: int, d: int, page: int = 64, device="cuda") -> torch.Tensor:
    """An empty pool of ``n_pages`` pages (its bytes are not initialised; nothing reads what was not written)."""
    if sa_cache_page_bytes(H, d, page) == 0:
        raise SketchError(2, "sa_cache_page_bytes")
    return torch.empty((n_pages, H, 2, page * (d // 2 + d // 16)), dtype=torch.uint8, device=device)


def _cache_args(pool, block_table, d: int):
    """(device index, n_pages, H, page, B, max_pages) after the checks that every cache call makes."""
    index = pool.get_device() if pool.is_cuda else -1
    if index < 0 or not pool.is_contiguous() or pool.dtype is not torch.uint8 or pool.dim() != 4:
        raise ValueError("pool must be a contiguous CUDA tensor, uint8 [n_pages, H, 2, page * (d/2 + d/16)]")
    if not block_table.is_cuda or block_table.get_device() != index or not block_table.is_contiguous() or \
            block_table.dtype is not torch.int32 or block_table.dim() != 2:
        raise ValueError("block_table must be contiguous int32 [B, max_pages] on the pool's device")
    n_pages, H, two, record = pool.shape
    page, rest = divmod(record * 16, 9 * d) if d > 0 else (0, 1)
    if two != 2 or rest:
        raise ValueError(f"a pool of shape {tuple(pool.shape)} holds no whole pages of rows of width {d}")
    B, max_pages = block_table.shape
    return index, n_pages, H, page, B, max_pages


def _offsets_arg(name, t, n, index):
    if t is None or not t.is_cuda or t.get_device() != index or t.dtype is not torch.int32 or t.dim() != 1 \
            or t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous int32 [{n}] on the pool's device")


def _ws_arg(ws, index):
    if not isinstance(ws, torch.Tensor) or not ws.is_cuda or ws.get_device() != index or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous tensor (uint8) on the pool's device")
    return ws


def sa_cache_write(pool: torch.Tensor, block_table: torch.Tensor, K: torch.Tensor, V: torch.Tensor,
                   cu_seqlens: Optional[torch.Tensor] = None, start: Optional[torch.Tensor] = None,
                   ws: Optional[torch.Tensor] = None, appends: bool = False) -> None:
    """Write rows into the cache in 4 bits: user b's row i to position start[b] + i.

    K, V are packed rows [N, H, d] with ``cu_seqlens`` [B+1], or [B, H, n, d] (a
    batch of sketches) without; fp32 or bf16, any strides with contiguous rows.

    To autograd this is an in-place change of the pool: the backward of an earlier
    ``sa_cache_attention`` over it is refused from then on.  ``appends`` is the caller's
    word that no such forward has seen the positions written, and leaves it allowed."""
    lib = load()
    packed = cu_seqlens is not None
    if K.dim() != (3 if packed else 4) or K.shape != V.shape or K.dtype != V.dtype:
        raise ValueError("K and V must be [N, H, d] with cu_seqlens, or [B, H, n, d] without, of one dtype")
    d = K.shape[-1]
    index, n_pages, H, page, B, max_pages = _cache_args(pool, block_table, d)
    if not K.is_cuda or K.get_device() != index or not V.is_cuda or V.get_device() != index:
        raise ValueError("K and V must be on the pool's device")
    if K.stride(-1) != 1 or V.stride() != K.stride():
        raise ValueError("K and V must have contiguous rows and equal strides")
    if K.shape[1] != H or (not packed and K.shape[0] != B):
        raise ValueError(f"K{tuple(K.shape)} does not fit a cache of {H} heads and {B} users")
    if start is not None:
        _offsets_arg("start", start, B, index)
    if packed:
        _offsets_arg("cu_seqlens", cu_seqlens, B + 1, index)
        N, strides = K.shape[0], (0, K.stride(0), K.stride(1))
    else:
        N, strides = B * K.shape[2], (K.stride(0), K.stride(2), K.stride(1))
    with _on(index):
        stream = _stream_handle(index)
        w = _ws_arg(ws, index) if ws is not None else _stream_workspace(256, index, stream)
        st = lib.sa_cache_write(K.data_ptr(), V.data_ptr(), *strides, _addr(cu_seqlens), B, N, _addr(start), H, d,
                                _dt(K), pool.data_ptr(), n_pages, page, block_table.data_ptr(), max_pages,
                                w.data_ptr(), w.numel(), stream)
    _check(st, "sa_cache_write")
    if not appends:
        torch.autograd.graph.increment_version(pool)
    if ws is None:
        _note_call(w, index, stream)


def sa_cache_read(pool: torch.Tensor, block_table: torch.Tensor, cu_seqlens: torch.Tensor, n_rows: int, d: int,
                  start: Optional[torch.Tensor] = None, dtype=torch.bfloat16, ws: Optional[torch.Tensor] = None):
    """(K, V) [n_rows, H, d]: positions start[b] .. of every user, n_rows = cu_seqlens[B] in all."""
    lib = load()
    index, n_pages, H, page, B, max_pages = _cache_args(pool, block_table, d)
    _offsets_arg("cu_seqlens", cu_seqlens, B + 1, index)
    if start is not None:
        _offsets_arg("start", start, B, index)
    if n_rows < 0:
        raise ValueError("n_rows must not be negative")
    K = torch.empty((n_rows, H, d), dtype=dtype, device=pool.device)
    V = torch.empty_like(K)
    with _on(index):
        stream = _stream_handle(index)
        w = _ws_arg(ws, index) if ws is not None else _stream_workspace(256, index, stream)
        st = lib.sa_cache_read(pool.data_ptr(), n_pages, page, block_table.data_ptr(), max_pages,
                               cu_seqlens.data_ptr(), B, n_rows, _addr(start), H, d, _dt(K), K.data_ptr(),
                               V.data_ptr(), w.data_ptr(), w.numel(), stream)
    _check(st, "sa_cache_read")
    if ws is None:
        _note_call(w, index, stream)
    return K, V


@functools.lru_cache(maxsize=1024)
def _attn_workspace_size(index: int, *sizes) -> int:
    """The size on device ``index``, which is current."""
    return int(load().sa_cache_attn_workspace_size(*sizes))


def sa_cache_attn_workspace_size(B: int, T: int, Hq: int, H: int, d: int, dt: int, max_tokens: int, bwd: bool) -> int:
    """Bytes of workspace that an attention call (``bwd``: its gradient) of these sizes needs on the current device."""
    return int(load().sa_cache_attn_workspace_size(B, T, Hq, H, d, dt, max_tokens, int(bool(bwd))))


def sa_cache_attn_kernel_name(B: int, T: int, Hq: int, H: int, d: int, scale: float, dt: int, bwd: bool) -> str:
    return load().sa_cache_attn_kernel_name(B, T, Hq, H, d, float(scale), dt, int(bool(bwd))).decode()


def _cache_attn(entry, q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale, ws, bwd: bool, *tensors):
    """What both directions check and pass; ``tensors``: the entry point's own."""
    if q.dim() != 3 or not q.is_cuda or q.stride(-1) != 1:
        raise ValueError("q must be a CUDA tensor [T, Hq, d] with contiguous rows")
    T, Hq, d = q.shape
    index, n_pages, H, page, B, max_pages = _cache_args(pool, block_table, d)
    if q.get_device() != index:
        raise ValueError("q must be on the pool's device")
    if Hq % H:
        raise ValueError(f"{Hq} query heads over {H} cached heads")
    _offsets_arg("cu_q", cu_q, B + 1, index)
    _offsets_arg("cache_lens", cache_lens, B, index)
    if kv_begin is not None:
        _offsets_arg("kv_begin", kv_begin, T, index)
    if kv_end is not None:
        _offsets_arg("kv_end", kv_end, T, index)
    dt = _dt(q)
    scale = 1.0 / math.sqrt(d) if scale is None else float(scale)
    with _on(index):
        stream = _stream_handle(index)
        if ws is not None:
            w = _ws_arg(ws, index)
        else:
            need = _attn_workspace_size(index, B, T, Hq, H, d, dt, max_pages * page, int(bwd))
            if need == 0:
                raise SketchError(2, "sa_cache_attn_workspace_size")
            w = _stream_workspace(need, index, stream)
        row, head, _ = q.stride()
        st = entry(q.data_ptr(), row, head, cu_q.data_ptr(), B, T, Hq, pool.data_ptr(), n_pages, page,
                   block_table.data_ptr(), max_pages, cache_lens.data_ptr(), H, d, _addr(kv_begin), _addr(kv_end),
                   scale, dt, *[_addr(t) for t in tensors], w.data_ptr(), w.numel(), stream)
    _check(st, "sa_cache_attn_bwd" if bwd else "sa_cache_attn_fwd")
    if ws is None:
        _note_call(w, index, stream)


def sa_cache_attn_fwd(q: torch.Tensor, cu_q: torch.Tensor, pool: torch.Tensor, block_table: torch.Tensor,
                      cache_lens: torch.Tensor, kv_begin: Optional[torch.Tensor] = None,
                      kv_end: Optional[torch.Tensor] = None, scale: Optional[float] = None, want_lse: bool = False,
                      ws: Optional[torch.Tensor] = None):
    """Attention of packed queries q [T, Hq, d] (user b's are cu_q[b] .. cu_q[b+1]-1) over the cache:
    out [T, Hq, d] like q (and lse [T, Hq] fp32).  Query t sees positions kv_begin[t] <= i < kv_end[t] below
    cache_lens[b] (all of them by default); one that sees nothing gets zeros and -inf."""
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device) if want_lse else None
    _cache_attn(load().sa_cache_attn_fwd, q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale, ws, False,
                out, lse)
    return (out, lse) if want_lse else out


def sa_cache_attn_bwd(q: torch.Tensor, cu_q: torch.Tensor, pool: torch.Tensor, block_table: torch.Tensor,
                      cache_lens: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                      kv_begin: Optional[torch.Tensor] = None, kv_end: Optional[torch.Tensor] = None,
                      scale: Optional[float] = None, ws: Optional[torch.Tensor] = None):
    """dq [T, Hq, d] like q for the gradient dout of ``sa_cache_attn_fwd``'s out; out and lse are that call's.
    The cached rows are constants and get no gradient."""
    for name, t, shape, dtype in (("out", out, q.shape, q.dtype), ("dout", dout, q.shape, q.dtype),
                                  ("lse", lse, q.shape[:2], torch.float32)):
        if t.shape != shape or t.dtype is not dtype or not t.is_contiguous() or t.get_device() != q.get_device():
            raise ValueError(f"{name} must be contiguous {dtype} {tuple(shape)} on q's device")
    dq = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _cache_attn(load().sa_cache_attn_bwd, q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale, ws, True,
                out, lse, dout, dq)
    return dq


class CacheAttention(torch.autograd.Function):
    """out = softmax(scale q K^T) V over each user's cached rows; gradient for q only, and once."""

    @staticmethod
    def forward(ctx, q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale):
        out, lse = sa_cache_attn_fwd(q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale, want_lse=True)
        ctx.save_for_backward(q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, out, lse)
        ctx.scale = scale
        return out

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dout):
        q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, out, lse = ctx.saved_tensors
        dq = sa_cache_attn_bwd(q, cu_q, pool, block_table, cache_lens, out, lse, dout.contiguous(), kv_begin, kv_end,
                               ctx.scale)
        return dq, None, None, None, None, None, None, None


def sa_cache_attention(q, cu_q, pool, block_table, cache_lens, kv_begin=None, kv_end=None,
                       scale: Optional[float] = None):
    """Differentiable (in q) attention of packed queries over the 4-bit cache: [T, Hq, d]."""
    return CacheAttention.apply(q, cu_q, pool, block_table, cache_lens, kv_begin, kv_end, scale)


# ------------------------------------------- layer norm and linear layers
# (include/sa_dense.h).  Rows are a tensor's last axis; the axes before it may have any shape
# whose rows lie a constant distance apart.

SA_ACT = {"none": 0, "relu": 1, "gelu": 2, "silu": 3, "swiglu": 4}

# Workspaces of these calls, apart from the cache's: reading one family's status must not depend on the other's calls.
_dense_ws = threading.local()
_dense_ws_cache = {}
# Larger ones (a gradient's dz, copies of operands) are taken from torch's allocator for each call and given back with the
# next on the stream: such a call takes tens of microseconds, an allocation two.
_DENSE_KEPT = 32 << 20


def sa_linear_get_device_error(device=None) -> int:
    """Status of the latest sa_linear_* call on the current stream (from any thread) that was given no ``ws``: 0, or
    SA_ERR_TIMEOUT where a wait gave up.  As ``sa_cache_get_device_error`` otherwise."""
    return _kept_status(device, _dense_ws_cache)


def _row_stride(name: str, t: torch.Tensor, n: int, index: int, dtype=None) -> int:
    """Elements between the rows of ``t`` [..., n] (its last axis contiguous)."""
    if t.get_device() != index:
        raise ValueError(f"{name} must be a CUDA tensor on the call's device")
    if t.dim() < 1 or t.shape[-1] != n or (dtype is not None and t.dtype is not dtype):
        raise ValueError(f"{name} must be {dtype or 'bf16 or fp32'} [..., {n}], not {t.dtype} {tuple(t.shape)}")
    if t.is_contiguous():
        return n
    if n > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    stride = rows = None
    for size, step in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size == 1:
            continue
        if stride is None:
            stride, rows = step, size
        elif step != stride * rows:
            raise ValueError(f"{name}'s rows must lie a constant distance apart")
        else:
            rows *= size
    return n if stride is None else stride


def _vector(name: str, t: Optional[torch.Tensor], n: int, index: int, dtype) -> Optional[int]:
    if t is None:
        return None
    if t.get_device() != index or t.dtype is not dtype or t.shape != (n,) or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous {dtype} [{n}] on the call's device")
    return t.data_ptr()


def _on_device(name: str, t: torch.Tensor) -> int:
    index = t.get_device()
    if index < 0 or not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    return index


def sa_layer_norm_fwd(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
                      residual: Optional[torch.Tensor] = None, eps: float = 1e-5, dtype=None,
                      want_stats: bool = False):
    """Layer norm over the last axis of x + residual: y [..., n] of ``dtype`` (x's by default), and with
    ``want_stats`` the rows' (mean, 1/sqrt(var + eps)), fp32 [..., 2], which the gradient takes.  x, residual,
    the parameters (of one type) and y are bf16 or fp32 each."""
    index = _on_device("x", x)
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return sa_layer_norm_fwd(x, weight, bias, residual, eps, dtype, want_stats)
    shape = x.shape
    if not shape:
        raise ValueError("x must be [..., n]")
    n = shape[-1]
    xs, rs, r_dt = _row_stride("x", x, n, index), 0, 0
    if residual is not None:
        if residual.shape != shape:
            raise ValueError(f"residual{tuple(residual.shape)} must have the shape of x{tuple(shape)}")
        rs, r_dt = _row_stride("residual", residual, n, index), _dt(residual)
    w_t = weight.dtype if weight is not None else bias.dtype if bias is not None else torch.float32
    w, b = _vector("weight", weight, n, index, w_t), _vector("bias", bias, n, index, w_t)
    device = x.device
    y = torch.empty(shape, dtype=x.dtype if dtype is None else dtype, device=device)
    stats = torch.empty((*shape[:-1], 2), dtype=torch.float32, device=device) if want_stats else None
    st = load().sa_layer_norm_fwd(x.data_ptr(), xs, _dt(x), _addr(residual), rs, r_dt, w, b, _dt_of(w_t),
                                  x.numel() // max(n, 1), n, eps, y.data_ptr(), _dt(y), _addr(stats),
                                  _stream_handle(index))
    if st:
        raise SketchError(st, "sa_layer_norm_fwd")
    return (y, stats) if want_stats else y


def _dt_of(dtype) -> int:
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype} (bf16 or fp32)")
    return SA_BF16 if dtype is torch.bfloat16 else SA_F32


def sa_layer_norm_bwd(dy: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, weight: Optional[torch.Tensor] = None,
                      residual: Optional[torch.Tensor] = None, want_dx: bool = True, want_params: bool = True,
                      ws: Optional[torch.Tensor] = None):
    """(dx, dr, dw, db) for the gradient dy of ``sa_layer_norm_fwd``'s y; ``stats`` are that call's.  dx is of x's
    type and dr of residual's (the same tensor where the types agree, None without a residual); dw and db [n] are of
    weight's type (fp32 without one).  What is not wanted is None."""
    index = _on_device("x", x)
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return sa_layer_norm_bwd(dy, x, stats, weight, residual, want_dx, want_params, ws)
    if x.dim() < 1 or dy.shape != x.shape:
        raise ValueError(f"dy{tuple(dy.shape)} must have the shape of x{tuple(x.shape)}, [..., n]")
    n = x.shape[-1]
    xs, ys = _row_stride("x", x, n, index), _row_stride("dy", dy, n, index)
    rs, r_dt = 0, 0
    if residual is not None:
        if residual.shape != x.shape:
            raise ValueError(f"residual{tuple(residual.shape)} must have the shape of x{tuple(x.shape)}")
        rs, r_dt = _row_stride("residual", residual, n, index), _dt(residual)
    if not stats.is_cuda or stats.get_device() != index or stats.dtype is not torch.float32 or \
            tuple(stats.shape) != (*x.shape[:-1], 2) or not stats.is_contiguous():
        raise ValueError(f"stats must be contiguous fp32 {(*x.shape[:-1], 2)} on x's device")
    w_t = weight.dtype if weight is not None else torch.float32
    w = _vector("weight", weight, n, index, w_t)
    rows = x.numel() // max(n, 1)
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device) if want_dx else None
    dr = None
    if residual is not None and want_dx:
        dr = dx if residual.dtype is x.dtype else torch.empty(x.shape, dtype=residual.dtype, device=x.device)
    dw = torch.empty(n, dtype=w_t, device=x.device) if want_params else None
    db = torch.empty(n, dtype=w_t, device=x.device) if want_params else None
    stream, at, size = _stream_handle(index), None, 0
    if want_params:
        need = _norm_workspace_size(index, rows, n)
        if need == 0:
            raise SketchError(2, "sa_layer_norm_workspace_size")
        w_buf = _ws_arg(ws, index) if ws is not None else _stream_workspace(need, index, stream, _dense_ws)
        at, size = w_buf.data_ptr(), w_buf.numel() * w_buf.element_size()
    st = load().sa_layer_norm_bwd(dy.data_ptr(), ys, _dt(dy), x.data_ptr(), xs, _dt(x), _addr(residual), rs, r_dt, w,
                                  _dt_of(w_t), stats.data_ptr(), rows, n, _addr(dx), None if dr is dx else _addr(dr),
                                  _addr(dw), _addr(db), at, size, stream)
    _check(st, "sa_layer_norm_bwd")
    return dx, dr, dw, db


@functools.lru_cache(maxsize=1024)
def _norm_workspace_size(index: int, rows: int, n: int) -> int:
    """The size on device ``index``, which is current."""
    return int(load().sa_layer_norm_workspace_size(rows, n))


def _gradient_follows(*tensors) -> bool:
    """Whether autograd records a call of these.  (Inside a Function's forward, where gradients are off, a parameter counts
    as needing one under ``torch.no_grad()`` too.)"""
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


class LayerNorm(torch.autograd.Function):
    """y = LN(x + residual) weight + bias over the last axis; differentiable once."""

    @staticmethod
    def forward(ctx, x, weight, bias, residual, eps, dtype):
        y, stats = sa_layer_norm_fwd(x, weight, bias, residual, eps, dtype, want_stats=True)
        ctx.save_for_backward(x, weight, bias, residual, stats)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, bias, residual, stats = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx, dr, dw, db = sa_layer_norm_bwd(dy.contiguous(), x, stats, weight, residual, need[0] or need[3],
                                           need[1] or need[2])
        if db is not None and bias is not None:
            db = db.to(bias.dtype)
        return dx if need[0] else None, dw if need[1] else None, db if need[2] else None, dr if need[3] else None, \
            None, None


def sa_layer_norm(x, weight=None, bias=None, residual=None, eps: float = 1e-5, dtype=None):
    """Differentiable layer norm of x + residual over the last axis, [..., n] of ``dtype`` (x's by default)."""
    if not _gradient_follows(x, weight, bias, residual):
        return sa_layer_norm_fwd(x, weight, bias, residual, eps, dtype)
    return LayerNorm.apply(x, weight, bias, residual, eps, dtype)


def _act(activation: Optional[str]) -> int:
    code = SA_ACT.get("none" if activation is None else activation)
    if code is None:
        raise ValueError(f"unknown activation {activation!r}: one of {', '.join(SA_ACT)}")
    return code


def _repack(t: torch.Tensor, stride: int, n: int) -> bool:
    return t.data_ptr() % 16 != 0 or stride * t.element_size() % 16 != 0 or stride < n


@functools.lru_cache(maxsize=1024)
def _linear_workspace_size(index: int, *sizes) -> int:
    """The size on device ``index``, which is current."""
    return int(load().sa_linear_workspace_size(*sizes))


def sa_linear_kernel_name(M: int, N: int, K: int, activation: Optional[str], dt: int, which: int) -> str:
    return load().sa_linear_kernel_name(M, N, K, _act(activation), dt, which).decode()


def _linear_args(x, weight, activation, index):
    act = _act(activation)
    if weight.dim() != 2 or x.dim() < 1 or weight.dtype is not x.dtype:
        raise ValueError("want x [..., K] and weight [N, K] (swiglu: [2 N, K]) of one dtype")
    Z, K = weight.shape
    if act == 4 and Z % 2:
        raise ValueError("swiglu takes a weight [2 N, K], the gate's N rows first")
    xs, wt = _row_stride("x", x, K, index), _row_stride("weight", weight, K, index)
    copies = _repack(x, xs, K) + 2 * _repack(weight, wt, K)
    return act, _dt(x), x.numel() // max(K, 1), Z // 2 if act == 4 else Z, Z, K, xs, wt, copies


def _linear_workspace(ws, index: int, stream: int, *sizes) -> torch.Tensor:
    if ws is not None:
        return _ws_arg(ws, index)
    need = _linear_workspace_size(index, *sizes)
    if need == 0:
        raise SketchError(2, "sa_linear_workspace_size")
    if need > _DENSE_KEPT:
        with _ws_lock:
            _dense_ws_cache.pop((index, stream), None)  # the last call's, whose status this call's replaces
        return torch.empty(need, dtype=torch.uint8, device=torch.device("cuda", index))
    return _stream_workspace(need, index, stream, _dense_ws)


def sa_linear_fwd(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None,
                  activation: Optional[str] = None, residual: Optional[torch.Tensor] = None, want_pre: bool = False,
                  ws: Optional[torch.Tensor] = None):
    """y = act(x weight^T + bias) + residual, [..., N] of x's type: x [..., K], weight [Z, K], bias [Z], residual
    [..., N].  ``activation``: none, relu, gelu (with the normal distribution function), silu, or swiglu, where the
    weight's first half of the rows makes the gate: silu(first) * second, N = Z / 2; else N = Z.  With ``want_pre``
    also what the activation is taken of, [..., Z], which the gradient takes (None for no activation)."""
    index = _on_device("x", x)
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return sa_linear_fwd(x, weight, bias, activation, residual, want_pre, ws)
    act, dt, M, N, Z, K, xs, wt, copies = _linear_args(x, weight, activation, index)
    lead, dtype, device = x.shape[:-1], x.dtype, x.device
    b, rs = _vector("bias", bias, Z, index, dtype), 0
    if residual is not None:
        if residual.shape != (*lead, N):
            raise ValueError(f"residual{tuple(residual.shape)} must be {(*lead, N)}")
        rs = _row_stride("residual", residual, N, index, dtype)
    y = torch.empty((*lead, N), dtype=dtype, device=device)
    z = torch.empty((*lead, Z), dtype=dtype, device=device) if want_pre and act else None
    stream = _stream_handle(index)
    w = _linear_workspace(ws, index, stream, M, N, K, act, dt, 0, copies)
    st = load().sa_linear_fwd(x.data_ptr(), xs, weight.data_ptr(), wt, b, _addr(residual), rs, M, N, K, act, dt,
                              y.data_ptr(), _addr(z), w.data_ptr(), w.nbytes, stream)
    if st:
        raise SketchError(st, "sa_linear_fwd")
    if ws is None:
        _note_call(w, index, stream, _dense_ws_cache)
    return (y, z) if want_pre else y


def sa_linear_bwd(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, pre: Optional[torch.Tensor] = None,
                  activation: Optional[str] = None, want_dx: bool = True, want_dw: bool = True, want_db: bool = True,
                  ws: Optional[torch.Tensor] = None):
    """(dx [..., K], dw [Z, K], db [Z]) of x's type for the gradient dy [..., N] of ``sa_linear_fwd``'s y; ``pre`` is
    that call's.  The residual's gradient is dy itself.  What is not wanted is None."""
    index = _on_device("x", x)
    if torch.cuda.current_device() != index:
        with torch.cuda.device(index):
            return sa_linear_bwd(dy, x, weight, pre, activation, want_dx, want_dw, want_db, ws)
    act, dt, M, N, Z, K, xs, wt, copies = _linear_args(x, weight, activation, index)
    lead, dtype, device = x.shape[:-1], x.dtype, x.device
    if dy.shape != (*lead, N):
        raise ValueError(f"dy{tuple(dy.shape)} must be {(*lead, N)}")
    ys = _row_stride("dy", dy, N, index, dtype)
    if act:
        if pre is None or pre.shape != (*lead, Z) or pre.dtype is not dtype or not pre.is_contiguous() or \
                pre.get_device() != index:
            raise ValueError(f"pre must be contiguous {dtype} {(*lead, Z)} on x's device")
    dx = torch.empty(x.shape, dtype=dtype, device=device) if want_dx else None
    dw = torch.empty((Z, K), dtype=dtype, device=device) if want_dw else None
    db = torch.empty(Z, dtype=dtype, device=device) if want_db else None
    stream = _stream_handle(index)
    w = _linear_workspace(ws, index, stream, M, N, K, act, dt, 1, copies + 4 * _repack(dy, ys, N))
    st = load().sa_linear_bwd(dy.data_ptr(), ys, x.data_ptr(), xs, weight.data_ptr(), wt, _addr(pre) if act else None,
                              M, N, K, act, dt, _addr(dx), _addr(dw), _addr(db), w.data_ptr(), w.nbytes, stream)
    _check(st, "sa_linear_bwd")
    if ws is None:
        _note_call(w, index, stream, _dense_ws_cache)
    return dx, dw, db


class Linear(torch.autograd.Function):
    """y = act(x weight^T + bias) + residual; differentiable once."""

    @staticmethod
    def forward(ctx, x, weight, bias, activation, residual):
        need = any(ctx.needs_input_grad[:3])
        y, pre = sa_linear_fwd(x, weight, bias, activation, residual, want_pre=need) if need else \
            (sa_linear_fwd(x, weight, bias, activation, residual), None)
        ctx.save_for_backward(x, weight, pre)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, pre = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw = db = None
        if any(need[:3]):
            dx, dw, db = sa_linear_bwd(dy.contiguous(), x, weight, pre, ctx.activation, *need[:3])
        return dx, dw, db, None, dy if need[4] else None


def sa_linear(x, weight, bias=None, activation: Optional[str] = None, residual=None):
    """Differentiable act(x weight^T + bias) + residual (see ``sa_linear_fwd``)."""
    if not _gradient_follows(x, weight, bias, residual):
        return sa_linear_fwd(x, weight, bias, activation, residual)
    return Linear.apply(x, weight, bias, activation, residual)
