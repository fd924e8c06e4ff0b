"""Thin Python binding of libebd (include/ebd.h): argument marshalling only.

Each function carries the name of the C entry point it calls and takes torch
tensors that already live on the GPU (the eviction calls also take K, V and
the scores as page-locked CPU tensors: the library then reads the scores and
only the kept rows from host memory); it checks shapes, dtypes and
contiguity, passes raw pointers plus sizes, and raises ``EbdError`` on a
non-OK status.  Every step of the hot path runs in the library's CUDA
kernels.  PyTorch supplies device memory and the current stream.  The calls of
a speculative serving step go through a C++ extension that makes the same checks
(csrc/binding.cpp); the others through ctypes.

If the compiled library is missing the import of any entry point raises: there
is no fallback implementation.
"""
from __future__ import annotations

import ctypes
import importlib.machinery
import importlib.util
import math
import os
from dataclasses import dataclass

import torch

from .build import CALL, LIB

__all__ = [
    "EbdError", "EbdDesign", "EBD_F32", "EBD_BF16", "EBD_RANGE_BOUND", "EBD_RANGE_EXACT",
    "EBD_DEV_CAPACITY", "EBD_DEV_NONFINITE", "EBD_DEV_TIMEOUT", "EBD_SAMPLING_POISSON",
    "EBD_SAMPLING_SYSTEMATIC", "lib", "lib_path",
    "ebd_status_string", "ebd_abi_version", "ebd_philox_uniforms", "ebd_score_workspace_bytes",
    "ebd_score", "ebd_compute_pi", "ebd_evict_workspace_bytes", "ebd_evict", "ebd_select",
    "ebd_gather", "ebd_decode_workspace_bytes", "ebd_workspace_bytes", "ebd_certified_decode",
    "ebd_certified_decode_static", "ebd_certificate_update", "ebd_append", "ebd_reevict",
    "ebd_gather_queries", "ebd_variance_contributions", "ebd_block_scores",
    "ebd_check_stalled_wait", "design_for",
    "CompactCache",
    "alloc_compact", "ABI_FUNCTIONS",
    "EBD_DEV_RANGE", "EBD_ROTARY_HALF", "EBD_ROTARY_PAIRS", "EbdPagedCache", "PagedCache",
    "alloc_paged", "rotary_frequencies", "ebd_rotary_table", "ebd_rotary", "ebd_paged_append",
    "ebd_paged_attention_workspace_bytes", "ebd_paged_attention", "ebd_paged_gather",
    "PagePool", "alloc_page_pool", "ebd_paged_deal", "ebd_norm_rotary",
    "ebd_norm_rotary_backward_workspace_bytes", "ebd_norm_rotary_backward",
    "ebd_paged_append_norm", "ebd_tree_masks", "ebd_paged_tree_attention", "ebd_paged_keep",
]

EBD_OK = 0
EBD_F32, EBD_BF16 = 0, 1
EBD_RANGE_BOUND, EBD_RANGE_EXACT = 0, 1
EBD_DEV_CAPACITY, EBD_DEV_NONFINITE, EBD_DEV_TIMEOUT = 0x1, 0x2, 0x4
EBD_SAMPLING_POISSON, EBD_SAMPLING_SYSTEMATIC = 0, 1
EBD_DEV_RANGE = 0x8
EBD_ROTARY_HALF, EBD_ROTARY_PAIRS = 0, 1

# Every symbol include/ebd.h declares.
ABI_FUNCTIONS = (
    "ebd_status_string", "ebd_abi_version", "ebd_philox_uniforms", "ebd_score_workspace_bytes",
    "ebd_score", "ebd_compute_pi", "ebd_evict_workspace_bytes", "ebd_evict", "ebd_select",
    "ebd_gather", "ebd_decode_workspace_bytes", "ebd_workspace_bytes", "ebd_certified_decode",
    "ebd_certified_decode_static", "ebd_certificate_update", "ebd_append", "ebd_reevict",
    "ebd_gather_queries", "ebd_variance_contributions", "ebd_block_scores",
    "ebd_check_stalled_wait", "ebd_rotary_table", "ebd_rotary", "ebd_paged_append",
    "ebd_paged_attention_workspace_bytes", "ebd_paged_attention", "ebd_paged_gather",
    "ebd_paged_deal", "ebd_norm_rotary", "ebd_norm_rotary_backward_workspace_bytes",
    "ebd_norm_rotary_backward", "ebd_paged_append_norm", "ebd_tree_masks",
    "ebd_paged_tree_attention", "ebd_paged_keep",
)


class EbdError(RuntimeError):
    def __init__(self, func: str, code: int, msg: str):
        super().__init__(f"{func} failed: {msg} (status {code})")
        self.code = code


class EbdDesign(ctypes.Structure):
    """Mirror of ``ebd_design`` in include/ebd.h."""
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("group", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("n_ctx", ctypes.c_int32), ("layer", ctypes.c_int32),
        ("seed", ctypes.c_uint64), ("n_sink", ctypes.c_int32), ("n_recent", ctypes.c_int32),
        ("k_head", ctypes.c_int32), ("budget_tokens", ctypes.c_int32),
        ("bisect_iters", ctypes.c_int32), ("eps", ctypes.c_float), ("sampling", ctypes.c_int32),
    ]


class EbdPagedCache(ctypes.Structure):
    """Mirror of ``ebd_paged_cache`` in include/ebd.h."""
    _fields_ = [
        ("dtype", ctypes.c_int32), ("batch", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32), ("n_pages", ctypes.c_int32),
        ("max_blocks", ctypes.c_int32), ("reserved", ctypes.c_int32),
        ("page_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64), ("K_pages", ctypes.c_void_p),
        ("V_pages", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
        ("seq_len", ctypes.c_void_p),
    ]


_LIB = None


def lib_path() -> str:
    return LIB


def lib():
    """Load libebd.so once; raise if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB):
            raise RuntimeError(f"{LIB} is not built; run `python -c \"import __graft_entry__ as g; "
                               f"g.build()\"` (no CPU fallback exists)")
        L = ctypes.CDLL(LIB)
        c_void_p, i32, u64, f32, sz = (ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64,
                                       ctypes.c_float, ctypes.c_size_t)
        i64, f64 = ctypes.c_int64, ctypes.c_double
        P = ctypes.POINTER(EbdDesign)
        C = ctypes.POINTER(EbdPagedCache)
        sig = {
            "ebd_status_string": (ctypes.c_char_p, [ctypes.c_int]),
            "ebd_abi_version": (i32, []),
            "ebd_philox_uniforms": (ctypes.c_int, [u64, i32, i32, i32, i32, c_void_p, c_void_p]),
            "ebd_score_workspace_bytes": (sz, [i32, i32, i32]),
            "ebd_score": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, i32, c_void_p, c_void_p,
                                         c_void_p, c_void_p, sz, c_void_p]),
            "ebd_compute_pi": (ctypes.c_int, [P, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
            "ebd_evict_workspace_bytes": (sz, [P, i32]),
            "ebd_evict": (ctypes.c_int, [P, ctypes.c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                         i32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, i32,
                                         c_void_p, c_void_p, sz, c_void_p]),
            "ebd_select": (ctypes.c_int, [P, c_void_p, c_void_p, c_void_p, c_void_p, i32, c_void_p,
                                          c_void_p]),
            "ebd_gather": (ctypes.c_int, [P, ctypes.c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                          i32, c_void_p, c_void_p, c_void_p]),
            "ebd_decode_workspace_bytes": (sz, [ctypes.c_int, i32, i32, i32, i32, i32]),
            "ebd_workspace_bytes": (sz, [P, i32]),
            "ebd_certified_decode": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, c_void_p,
                                                    c_void_p, c_void_p, c_void_p, c_void_p, i32,
                                                    f32, f32, ctypes.c_int, c_void_p, c_void_p,
                                                    c_void_p, c_void_p, c_void_p, c_void_p,
                                                    c_void_p, sz, c_void_p]),
            "ebd_certified_decode_static": (ctypes.c_int, [
                ctypes.c_int, i32, i32, i32, i32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                i32, f32, f32, ctypes.c_int, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                c_void_p, c_void_p]),
            "ebd_certificate_update": (ctypes.c_int, [c_void_p, i32, i32, i32, i32, f32, i32,
                                                      c_void_p, c_void_p, c_void_p, c_void_p]),
            "ebd_append": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, c_void_p, c_void_p,
                                          c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                          c_void_p, i32, c_void_p, c_void_p]),
            "ebd_reevict": (ctypes.c_int, [P, ctypes.c_int, c_void_p, c_void_p, c_void_p, c_void_p,
                                           c_void_p, c_void_p, i32, c_void_p, c_void_p, c_void_p,
                                           c_void_p, c_void_p, i32, c_void_p, c_void_p]),
            "ebd_gather_queries": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, i32, c_void_p,
                                                  c_void_p, i32, c_void_p, c_void_p]),
            "ebd_variance_contributions": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32,
                                                          c_void_p, c_void_p, c_void_p, c_void_p,
                                                          c_void_p, i32, c_void_p, c_void_p,
                                                          c_void_p, c_void_p]),
            "ebd_block_scores": (ctypes.c_int, [i32, i32, i32, c_void_p, c_void_p, c_void_p, i32,
                                                i32, i32, c_void_p, c_void_p]),
            "ebd_check_stalled_wait": (ctypes.c_int, [c_void_p, c_void_p]),
            "ebd_rotary_table": (ctypes.c_int, [c_void_p, i32, i32, f64, c_void_p, c_void_p]),
            "ebd_rotary": (ctypes.c_int, [ctypes.c_int, i32, i32, i32, i32, ctypes.c_int, i32,
                                          c_void_p, i64, i64, c_void_p, c_void_p, i32, c_void_p,
                                          i64, i64, c_void_p, c_void_p]),
            "ebd_paged_append": (ctypes.c_int, [C, i32, c_void_p, c_void_p, i64, i64, c_void_p,
                                                i64, i64, c_void_p, i32, i32, ctypes.c_int, i32,
                                                c_void_p, i64, i64, c_void_p, i64, i64, c_void_p,
                                                c_void_p]),
            "ebd_paged_attention_workspace_bytes": (sz, [C, i32, i32]),
            "ebd_paged_attention": (ctypes.c_int, [C, i32, i32, i32, c_void_p, c_void_p, i64, i64,
                                                   f32, i32, c_void_p, c_void_p, c_void_p,
                                                   c_void_p, sz, c_void_p]),
            "ebd_paged_gather": (ctypes.c_int, [C, c_void_p, c_void_p, i32, c_void_p, c_void_p,
                                                c_void_p, c_void_p]),
            "ebd_paged_deal": (ctypes.c_int, [i32] * 6 + [c_void_p] * 15),
            "ebd_norm_rotary": (ctypes.c_int, [
                ctypes.c_int, i32, i32, i32, c_void_p, i64, i64, c_void_p, ctypes.c_int, i64, f32,
                c_void_p, c_void_p, i32, i32, ctypes.c_int, c_void_p, i64, i64, c_void_p,
                c_void_p]),
            "ebd_norm_rotary_backward_workspace_bytes": (sz, [i32, i32, i32]),
            "ebd_norm_rotary_backward": (ctypes.c_int, [
                ctypes.c_int, i32, i32, i32, c_void_p, i64, i64, c_void_p, i64, i64, c_void_p,
                ctypes.c_int, i64, f32, c_void_p, c_void_p, i32, i32, ctypes.c_int, c_void_p, i64,
                i64, c_void_p, c_void_p, c_void_p, sz, c_void_p]),
            "ebd_paged_append_norm": (ctypes.c_int, [
                C, i32, c_void_p, c_void_p, c_void_p, c_void_p, i64, i64, c_void_p, i64, i64,
                c_void_p, i64, c_void_p, i64, ctypes.c_int, f32, c_void_p, i32, i32, ctypes.c_int,
                i32, c_void_p, i64, i64, c_void_p, i64, i64, c_void_p, c_void_p]),
            "ebd_tree_masks": (ctypes.c_int, [i32, i32, i32, c_void_p, c_void_p, c_void_p, i32,
                                              c_void_p, i32, c_void_p, c_void_p, c_void_p]),
            "ebd_paged_tree_attention": (ctypes.c_int, [
                C, i32, i32, i32, c_void_p, c_void_p, i64, i64, f32, i32, c_void_p, i32, c_void_p,
                c_void_p, c_void_p, c_void_p, c_void_p, sz, c_void_p]),
            "ebd_paged_keep": (ctypes.c_int, [C, i32, i64, c_void_p, c_void_p, i32, c_void_p,
                                              c_void_p, c_void_p, c_void_p]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = L
    return _LIB


_CALL = None


def _call():
    """The extension that marshals the serving calls (csrc/binding.cpp), bound to the
    library once; raises if it has not been built."""
    global _CALL
    if _CALL is None:
        L = lib()
        if not os.path.exists(CALL):
            raise RuntimeError(f"{CALL} is not built; run `python -c \"import __graft_entry__ as "
                               f"g; g.build()\"` (no fallback exists)")
        loader = importlib.machinery.ExtensionFileLoader("ebd_call", CALL)
        m = importlib.util.module_from_spec(importlib.util.spec_from_loader("ebd_call", loader))
        loader.exec_module(m)
        m.bind({name: ctypes.cast(getattr(L, name), ctypes.c_void_p).value
                for name in ABI_FUNCTIONS})
        _CALL = m
    return _CALL


# ----------------------------------------------------------------- helpers
def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return EBD_F32
    if t.dtype == torch.bfloat16:
        return EBD_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; expected float32 or bfloat16")


def _ptr(t, dtype=None, shape=None, name="tensor", host_ok=False):
    """Address of a contiguous tensor.  host_ok: a page-locked CPU tensor is
    accepted too (the library reads it from the device over the host link)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda and not (host_ok and t.is_pinned()):
        raise ValueError(f"{name} must be a CUDA tensor" +
                         (" or a page-locked CPU tensor" if host_ok else ""))
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if shape is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


# torch.cuda.current_stream() builds a Stream object (microseconds per call);
# the raw handle of the same stream is enough here
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _check(name, code):
    if code != EBD_OK:
        raise EbdError(name, code, ebd_status_string(code))


def _empty(shape, dtype, device, stream=None):
    """A buffer for a call on `stream` (None: the current one), from that stream's
    pool: the allocator hands out memory whose last use may still be queued on
    the pool's own stream, and takes it back for later work there."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _result(shape, dtype, device, stream=None):
    """The same for a tensor that is returned: the current stream may read it too."""
    t = _empty(shape, dtype, device, stream)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _on_device(t, device, stream=None):
    """t on `device`; a copy is ordered, and lives, on `stream`."""
    if stream is None:
        return t.to(device)
    with torch.cuda.stream(stream):
        return t.to(device)


def _workspace(nbytes, device, ws, stream=None):
    if nbytes == 0:
        return None, 0
    if ws is None:
        ws = _empty(nbytes, torch.uint8, device, stream)
    if ws.numel() * ws.element_size() < nbytes:
        raise ValueError(f"workspace too small: {ws.numel() * ws.element_size()} < {nbytes}")
    return ws.data_ptr(), ws.numel() * ws.element_size()


# ---------------------------------------------------------------- entry points
def ebd_status_string(code: int) -> str:
    return lib().ebd_status_string(int(code)).decode()


def ebd_abi_version() -> int:
    return int(lib().ebd_abi_version())


def ebd_check_stalled_wait(dev_status: torch.Tensor, stream=None) -> torch.Tensor:
    """Run the bounded-wait failure path: ~2 s later EBD_DEV_TIMEOUT is OR-ed
    into dev_status (int32 CUDA tensor [1]) and the context stays usable."""
    _check("ebd_check_stalled_wait", lib().ebd_check_stalled_wait(
        _ptr(dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return dev_status


def ebd_philox_uniforms(seed: int, layer: int, x0: torch.Tensor, stream=None):
    """x0: int32 CUDA tensor [B, Hkv, N], filled with the uint32 Philox words."""
    B, H, N = x0.shape
    _check("ebd_philox_uniforms", lib().ebd_philox_uniforms(
        int(seed), int(layer), B, H, N, _ptr(x0, torch.int32, name="x0"), _stream(stream)))
    return x0


def ebd_score_workspace_bytes(batch, n_kv_heads, n_obs) -> int:
    return int(lib().ebd_score_workspace_bytes(batch, n_kv_heads, n_obs))


def ebd_score(q_obs: torch.Tensor, K: torch.Tensor, scores: torch.Tensor, workspace=None,
              stream=None):
    B, H, N, d = K.shape
    R = q_obs.shape[2]
    dt = _dtype_code(K)
    ws, wsb = _workspace(ebd_score_workspace_bytes(B, H, R), K.device, workspace, stream)
    _check("ebd_score", lib().ebd_score(
        dt, B, H, d, N, R, _ptr(q_obs, K.dtype, (B, H, R, d), "q_obs"), _ptr(K, name="K"),
        _ptr(scores, torch.float32, (B, H, N), "scores"), ws, wsb, _stream(stream)))
    return scores


def design_for(*, batch, n_kv_heads, group, head_dim, n_ctx, layer=0, seed=0, n_sink=4,
               n_recent=32, k_head, budget_tokens, bisect_iters=40, eps=1e-6,
               sampling=0) -> EbdDesign:
    return EbdDesign(batch, n_kv_heads, group, head_dim, n_ctx, layer, seed, n_sink, n_recent,
                     k_head, budget_tokens, bisect_iters, eps, sampling)


def ebd_compute_pi(design: EbdDesign, scores: torch.Tensor, pi: torch.Tensor,
                   certain_mask=None, dev_status=None, stream=None):
    shp = (design.batch, design.n_kv_heads, design.n_ctx)
    _check("ebd_compute_pi", lib().ebd_compute_pi(
        ctypes.byref(design), _ptr(scores, torch.float32, shp, "scores", True),
        _ptr(pi, torch.float32, shp, "pi"), _ptr(certain_mask, torch.uint8, shp, "certain_mask"),
        _ptr(dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return pi


def ebd_evict_workspace_bytes(design: EbdDesign, n_obs: int) -> int:
    return int(lib().ebd_evict_workspace_bytes(ctypes.byref(design), int(n_obs)))


def ebd_workspace_bytes(design: EbdDesign, capacity: int) -> int:
    """One workspace size serving every call of a layer with this design."""
    return int(lib().ebd_workspace_bytes(ctypes.byref(design), int(capacity)))


@dataclass
class CompactCache:
    K_c: torch.Tensor      # [B, Hkv, cap, d]
    V_c: torch.Tensor      # [B, Hkv, cap, d]
    logw_c: torch.Tensor   # [B, Hkv, cap] float32
    idx_c: torch.Tensor    # [B, Hkv, cap] int32
    n_kept: torch.Tensor   # [B, Hkv] int32
    dev_status: torch.Tensor  # [1] int32

    @property
    def capacity(self) -> int:
        return self.K_c.shape[2]


def alloc_compact(batch, n_kv_heads, capacity, head_dim, dtype, device) -> CompactCache:
    """Caller-side allocation of the compact-cache buffers (plain torch.empty)."""
    return CompactCache(
        torch.empty((batch, n_kv_heads, capacity, head_dim), dtype=dtype, device=device),
        torch.empty((batch, n_kv_heads, capacity, head_dim), dtype=dtype, device=device),
        torch.empty((batch, n_kv_heads, capacity), dtype=torch.float32, device=device),
        torch.empty((batch, n_kv_heads, capacity), dtype=torch.int32, device=device),
        torch.empty((batch, n_kv_heads), dtype=torch.int32, device=device),
        torch.zeros((1,), dtype=torch.int32, device=device),
    )


def ebd_evict(design: EbdDesign, K: torch.Tensor, V: torch.Tensor, scores, q_obs,
              out: CompactCache, workspace=None, stream=None) -> CompactCache:
    B, H, N, d = design.batch, design.n_kv_heads, design.n_ctx, design.head_dim
    dt = _dtype_code(K)
    cap = out.capacity
    n_obs = 0 if q_obs is None else q_obs.shape[2]
    if scores is None and q_obs is None:
        raise ValueError("ebd_evict needs scores or q_obs")
    ws, wsb = (None, 0)
    if scores is None:
        ws, wsb = _workspace(ebd_evict_workspace_bytes(design, n_obs), K.device, workspace,
                             stream)
    host_ok = scores is not None  # K, V, scores may stay in page-locked host memory
    _check("ebd_evict", lib().ebd_evict(
        ctypes.byref(design), dt, _ptr(K, K.dtype, (B, H, N, d), "K", host_ok),
        _ptr(V, K.dtype, (B, H, N, d), "V", True),
        _ptr(scores, torch.float32, (B, H, N), "scores", True),
        _ptr(q_obs, K.dtype, None if q_obs is None else (B, H, n_obs, d), "q_obs"), n_obs,
        _ptr(out.K_c, K.dtype, (B, H, cap, d), "K_c"), _ptr(out.V_c, K.dtype, (B, H, cap, d), "V_c"),
        _ptr(out.logw_c, torch.float32, (B, H, cap), "logw_c"),
        _ptr(out.idx_c, torch.int32, (B, H, cap), "idx_c"),
        _ptr(out.n_kept, torch.int32, (B, H), "n_kept"), cap,
        _ptr(out.dev_status, torch.int32, (1,), "dev_status"), ws, wsb, _stream(stream)))
    return out


def ebd_select(design: EbdDesign, scores: torch.Tensor, out: CompactCache, stream=None):
    """Certainty set, pi, Poisson draw and index compaction (no row copy)."""
    B, H, N = design.batch, design.n_kv_heads, design.n_ctx
    cap = out.capacity
    _check("ebd_select", lib().ebd_select(
        ctypes.byref(design), _ptr(scores, torch.float32, (B, H, N), "scores", True),
        _ptr(out.idx_c, torch.int32, (B, H, cap), "idx_c"),
        _ptr(out.logw_c, torch.float32, (B, H, cap), "logw_c"),
        _ptr(out.n_kept, torch.int32, (B, H), "n_kept"), cap,
        _ptr(out.dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return out


def ebd_gather(design: EbdDesign, K: torch.Tensor, V: torch.Tensor, out: CompactCache,
               stream=None):
    """Copy the kept K/V rows named by out.idx_c into out.K_c / out.V_c."""
    B, H, N, d = design.batch, design.n_kv_heads, design.n_ctx, design.head_dim
    cap = out.capacity
    _check("ebd_gather", lib().ebd_gather(
        ctypes.byref(design), _dtype_code(K), _ptr(K, K.dtype, (B, H, N, d), "K", True),
        _ptr(V, K.dtype, (B, H, N, d), "V", True),
        _ptr(out.idx_c, torch.int32, (B, H, cap), "idx_c"),
        _ptr(out.n_kept, torch.int32, (B, H), "n_kept"), cap,
        _ptr(out.K_c, K.dtype, (B, H, cap, d), "K_c"), _ptr(out.V_c, K.dtype, (B, H, cap, d), "V_c"),
        _stream(stream)))
    return out


def ebd_decode_workspace_bytes(dtype_code, batch, n_kv_heads, group, head_dim, capacity) -> int:
    return int(lib().ebd_decode_workspace_bytes(dtype_code, batch, n_kv_heads, group, head_dim,
                                                capacity))


def ebd_certified_decode(Q: torch.Tensor, K_c: torch.Tensor, V_c: torch.Tensor,
                         logw_c: torch.Tensor, n_kept: torch.Tensor, y: torch.Tensor,
                         lse: torch.Tensor, var_hat: torch.Tensor, b_t: torch.Tensor,
                         radius: torch.Tensor, delta: float = 0.1, eps0: float = 1e-9,
                         range_mode: int = EBD_RANGE_BOUND, dev_status=None, workspace=None,
                         stream=None):
    B, H, cap, d = K_c.shape
    Hq = Q.shape[1]
    if Hq % H:
        raise ValueError("query heads must be a multiple of KV heads")
    G = Hq // H
    dt = _dtype_code(K_c)
    ws, wsb = _workspace(ebd_decode_workspace_bytes(dt, B, H, G, d, cap), K_c.device, workspace,
                         stream)
    f = torch.float32
    _check("ebd_certified_decode", lib().ebd_certified_decode(
        dt, B, H, G, d, _ptr(Q, K_c.dtype, (B, Hq, d), "Q"), _ptr(K_c, name="K_c"),
        _ptr(V_c, K_c.dtype, (B, H, cap, d), "V_c"), _ptr(logw_c, f, (B, H, cap), "logw_c"),
        _ptr(n_kept, torch.int32, (B, H), "n_kept"), cap, float(delta), float(eps0),
        int(range_mode), _ptr(y, f, (B, Hq, d), "y"), _ptr(lse, f, (B, Hq), "lse"),
        _ptr(var_hat, f, (B, Hq), "var_hat"), _ptr(b_t, f, (B, Hq), "b_t"),
        _ptr(radius, f, (B, Hq), "radius"), _ptr(dev_status, torch.int32, (1,), "dev_status"),
        ws, wsb, _stream(stream)))
    return y, lse, var_hat, b_t, radius


def ebd_certified_decode_static(Q: torch.Tensor, K_c: torch.Tensor, V_c: torch.Tensor,
                                logw_c: torch.Tensor, n_kept: torch.Tensor, y: torch.Tensor,
                                lse: torch.Tensor, var_hat: torch.Tensor, b_t: torch.Tensor,
                                radius: torch.Tensor, delta: float = 0.1, eps0: float = 1e-9,
                                range_mode: int = EBD_RANGE_BOUND, dev_status=None, stream=None):
    """ebd_certified_decode without a workspace: for callers that cannot allocate
    device memory, the library uses its own fixed 16 MiB scratch array."""
    B, H, cap, d = K_c.shape
    Hq = Q.shape[1]
    if Hq % H:
        raise ValueError("query heads must be a multiple of KV heads")
    G = Hq // H
    f = torch.float32
    _check("ebd_certified_decode_static", lib().ebd_certified_decode_static(
        _dtype_code(K_c), B, H, G, d, _ptr(Q, K_c.dtype, (B, Hq, d), "Q"), _ptr(K_c, name="K_c"),
        _ptr(V_c, K_c.dtype, (B, H, cap, d), "V_c"), _ptr(logw_c, f, (B, H, cap), "logw_c"),
        _ptr(n_kept, torch.int32, (B, H), "n_kept"), cap, float(delta), float(eps0),
        int(range_mode), _ptr(y, f, (B, Hq, d), "y"), _ptr(lse, f, (B, Hq), "lse"),
        _ptr(var_hat, f, (B, Hq), "var_hat"), _ptr(b_t, f, (B, Hq), "b_t"),
        _ptr(radius, f, (B, Hq), "radius"), _ptr(dev_status, torch.int32, (1,), "dev_status"),
        _stream(stream)))
    return y, lse, var_hat, b_t, radius


def ebd_certificate_update(radius: torch.Tensor, cert: torch.Tensor, first_step: bool,
                           head_stride: int = 4, tau: float = 1.0, step_mean=None, red_flag=None,
                           stream=None):
    """One probed decode step of the deployed certificate: radius [L, B, Hq]
    (this step's r_t of every layer) -> cert [B] = max over probed steps of the
    mean over layers and every `head_stride`-th head; red_flag [B] = cert >= tau."""
    L, B, Hq = radius.shape
    f = torch.float32
    _check("ebd_certificate_update", lib().ebd_certificate_update(
        _ptr(radius, f, (L, B, Hq), "radius"), L, B, Hq, int(head_stride), float(tau),
        1 if first_step else 0, _ptr(step_mean, f, (B,), "step_mean"), _ptr(cert, f, (B,), "cert"),
        _ptr(red_flag, torch.int32, (B,), "red_flag"), _stream(stream)))
    return cert


def ebd_append(cc: "CompactCache", k_new: torch.Tensor, v_new: torch.Tensor,
               positions: torch.Tensor, stream=None) -> "CompactCache":
    """Append one token per unit (pi = 1) to the compact cache `cc` in place.
    k_new, v_new: [B, Hkv, d]; positions: [B] int32 token positions."""
    B, H, cap, d = cc.K_c.shape
    dt = _dtype_code(cc.K_c)
    _check("ebd_append", lib().ebd_append(
        dt, B, H, d, _ptr(k_new, cc.K_c.dtype, (B, H, d), "k_new"),
        _ptr(v_new, cc.K_c.dtype, (B, H, d), "v_new"), _ptr(positions, torch.int32, (B,), "positions"),
        _ptr(cc.K_c, name="K_c"), _ptr(cc.V_c, cc.K_c.dtype, (B, H, cap, d), "V_c"),
        _ptr(cc.logw_c, torch.float32, (B, H, cap), "logw_c"),
        _ptr(cc.idx_c, torch.int32, (B, H, cap), "idx_c"),
        _ptr(cc.n_kept, torch.int32, (B, H), "n_kept"), cap,
        _ptr(cc.dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return cc


def ebd_reevict(design: EbdDesign, scores: torch.Tensor, cc_in: "CompactCache",
                out: "CompactCache", stream=None) -> "CompactCache":
    """Evict the resident cache `cc_in` again into `out` (distinct buffers):
    scores [B, Hkv, cap_in] for the resident rows; design.n_ctx == cap_in."""
    B, H, cap_in, d = cc_in.K_c.shape
    cap_out = out.K_c.shape[2]
    dt = _dtype_code(cc_in.K_c)
    f = torch.float32
    _check("ebd_reevict", lib().ebd_reevict(
        ctypes.byref(design), dt, _ptr(scores, f, (B, H, cap_in), "scores"),
        _ptr(cc_in.K_c, name="K_in"), _ptr(cc_in.V_c, cc_in.K_c.dtype, (B, H, cap_in, d), "V_in"),
        _ptr(cc_in.logw_c, f, (B, H, cap_in), "logw_in"),
        _ptr(cc_in.idx_c, torch.int32, (B, H, cap_in), "idx_in"),
        _ptr(cc_in.n_kept, torch.int32, (B, H), "n_kept_in"), cap_in,
        _ptr(out.K_c, cc_in.K_c.dtype, (B, H, cap_out, d), "K_out"),
        _ptr(out.V_c, cc_in.K_c.dtype, (B, H, cap_out, d), "V_out"),
        _ptr(out.logw_c, f, (B, H, cap_out), "logw_out"),
        _ptr(out.idx_c, torch.int32, (B, H, cap_out), "idx_out"),
        _ptr(out.n_kept, torch.int32, (B, H), "n_kept_out"), cap_out,
        _ptr(out.dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return out


def ebd_gather_queries(Q: torch.Tensor, positions: torch.Tensor, n_kv_heads: int,
                       q_obs=None, stream=None) -> torch.Tensor:
    """Observation rows for ebd_score from prefill queries Q [B, Hq, Nq, d] at
    positions [P] (int32, device): q_obs [B, Hkv, G*P, d], row g*P + p."""
    B, Hq, Nq, d = Q.shape
    if Hq % n_kv_heads:
        raise ValueError("query heads must be a multiple of KV heads")
    G = Hq // n_kv_heads
    P = positions.shape[0]
    if q_obs is None:
        q_obs = _result((B, n_kv_heads, G * P, d), Q.dtype, Q.device, stream)
    _check("ebd_gather_queries", lib().ebd_gather_queries(
        _dtype_code(Q), B, n_kv_heads, G, d, Nq, _ptr(Q, name="Q"),
        _ptr(positions, torch.int32, (P,), "positions"), P,
        _ptr(q_obs, Q.dtype, (B, n_kv_heads, G * P, d), "q_obs"), _stream(stream)))
    return q_obs


def ebd_variance_contributions(Q: torch.Tensor, K_c: torch.Tensor, V_c: torch.Tensor,
                               logw_c: torch.Tensor, n_kept: torch.Tensor, y: torch.Tensor,
                               lse: torch.Tensor, contrib=None, stream=None) -> torch.Tensor:
    """Theorem 2's per-token terms [B, Hq, cap] (they sum to V_hat per head)."""
    B, H, cap, d = K_c.shape
    Hq = Q.shape[1]
    G = Hq // H
    f = torch.float32
    if contrib is None:
        contrib = _result((B, Hq, cap), f, K_c.device, stream)
    _check("ebd_variance_contributions", lib().ebd_variance_contributions(
        _dtype_code(K_c), B, H, G, d, _ptr(Q, K_c.dtype, (B, Hq, d), "Q"), _ptr(K_c, name="K_c"),
        _ptr(V_c, K_c.dtype, (B, H, cap, d), "V_c"), _ptr(logw_c, f, (B, H, cap), "logw_c"),
        _ptr(n_kept, torch.int32, (B, H), "n_kept"), cap, _ptr(y, f, (B, Hq, d), "y"),
        _ptr(lse, f, (B, Hq), "lse"), _ptr(contrib, f, (B, Hq, cap), "contrib"), _stream(stream)))
    return contrib


def ebd_block_scores(contrib: torch.Tensor, idx_c: torch.Tensor, n_kept: torch.Tensor,
                     block: int, n_blocks: int, out=None, stream=None) -> torch.Tensor:
    """Sum of retained contributions per block of `block` original positions."""
    B, H, cap = idx_c.shape
    Hq = contrib.shape[1]
    G = Hq // H
    if out is None:
        out = _result((B, H, n_blocks), torch.float32, idx_c.device, stream)
    _check("ebd_block_scores", lib().ebd_block_scores(
        B, H, G, _ptr(contrib, torch.float32, (B, Hq, cap), "contrib"),
        _ptr(idx_c, torch.int32, (B, H, cap), "idx_c"), _ptr(n_kept, torch.int32, (B, H), "n_kept"),
        cap, int(block), int(n_blocks), _ptr(out, torch.float32, (B, H, n_blocks), "out"),
        _stream(stream)))
    return out


# ---------------------------------------------------------------- paged cache
@dataclass
class PagedCache:
    """A pool of pages and the block table that deals them to sequences.

    K_pages and V_pages are [n_pages, Hkv, page_size, d] tensors of equal
    strides with the last dimension contiguous (views of another order, such
    as ``pool.transpose(1, 2)`` of a [n_pages, page_size, Hkv, d] pool, serve
    as they are); block_table [B, max_blocks] and seq_len [B] are int32.
    seq_len counts the new tokens of the call it is passed to."""
    K_pages: torch.Tensor
    V_pages: torch.Tensor
    block_table: torch.Tensor
    seq_len: torch.Tensor
    dev_status: torch.Tensor  # [1] int32


def alloc_paged(batch, n_kv_heads, n_pages, page_size, head_dim, max_blocks, dtype,
                device) -> PagedCache:
    """Caller-side allocation of a paged cache: empty pages, an all-zero block
    table and lengths of zero."""
    shape = (n_pages, n_kv_heads, page_size, head_dim)
    i = torch.int32
    return PagedCache(torch.empty(shape, dtype=dtype, device=device),
                      torch.empty(shape, dtype=dtype, device=device),
                      torch.zeros((batch, max_blocks), dtype=i, device=device),
                      torch.zeros((batch,), dtype=i, device=device),
                      torch.zeros((1,), dtype=i, device=device))


def _paged(pc: PagedCache) -> EbdPagedCache:
    K, V, bt, n = pc.K_pages, pc.V_pages, pc.block_table, pc.seq_len
    shape, stride = K.shape, K.stride()
    if len(shape) != 4 or V.shape != shape or V.stride() != stride:
        raise ValueError("K_pages and V_pages must be [n_pages, Hkv, page_size, d] tensors of "
                         "equal shapes and strides")
    if not (K.is_cuda and V.is_cuda and bt.is_cuda and n.is_cuda):
        raise ValueError("a paged cache's tensors must be CUDA tensors")
    dt = K.dtype
    if V.dtype != dt:
        raise TypeError(f"V_pages has dtype {V.dtype}, expected {dt}")
    if bt.dtype != torch.int32 or n.dtype != torch.int32:
        raise TypeError("block_table and seq_len must be int32")
    if bt.dim() != 2 or n.dim() != 1 or bt.shape[0] != n.shape[0] or not (
            bt.is_contiguous() and n.is_contiguous()):
        raise ValueError("block_table must be a contiguous [B, max_blocks] and seq_len a "
                         "contiguous [B] tensor")
    B, blocks = bt.shape
    n_pages, H, page, d = shape
    ps, hs, rs, cs = stride
    if cs != 1:
        raise ValueError("the last dimension of K_pages and V_pages must be contiguous")
    return EbdPagedCache(_dtype_code(K), B, H, d, page, n_pages, blocks, 0, ps, hs, rs,
                         K.data_ptr(), V.data_ptr(), bt.data_ptr(), n.data_ptr())


def _rows(t, dtype, n_tokens, n_heads, head_dim, name):
    """(address, token stride, head stride) of a [T, H, d] tensor with any
    token and head strides."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if t.shape != (n_tokens, n_heads, head_dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected "
                         f"{(n_tokens, n_heads, head_dim)}")
    ts, hs, cs = t.stride()
    if cs != 1 and head_dim > 1:
        raise ValueError(f"the last dimension of {name} must be contiguous")
    return t.data_ptr(), ts, hs


def _rotary_rows(table):
    if table.dim() != 3 or table.shape[2] != 2:
        raise ValueError(f"table has shape {tuple(table.shape)}, expected [n_pos, rotary_dim / 2, 2]")
    return _ptr(table, torch.float32, name="table"), table.shape[0], 2 * table.shape[1]


def rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none",
                       factor: float = 1.0, original_positions: int = 4096,
                       fast_turns: float = 32.0, slow_turns: float = 1.0):
    """(inv_freq [rotary_dim / 2] float64 on the CPU, mscale) for
    ``ebd_rotary_table``: f_i = base^(-2i / R), and for contexts `factor` times
    the original length

    - "linear": every f_i / factor (positions compressed);
    - "base": base * factor^(R / (R - 2)): the slowest pair slows by `factor`,
      the fastest stays;
    - "parts": a pair that makes at least `fast_turns` turns over
      `original_positions` stays, one that makes at most `slow_turns` slows by
      `factor`, in between the two are mixed linearly in the pair's index, from the
      last index that stays to the first that slows in full (either may lie
      outside 0 .. R / 2 - 1); the table grows by mscale = 0.1 ln(factor) + 1."""
    if rotary_dim < 2 or rotary_dim % 2:
        raise ValueError("rotary_dim must be even and at least 2")
    if not base > 1 or not factor >= 1:
        raise ValueError("base must be above 1 and factor at least 1")
    if scaling not in ("none", "linear", "base", "parts"):
        raise ValueError(f"unknown scaling {scaling!r}")
    if scaling == "base" and rotary_dim > 2:
        base = base * factor ** (rotary_dim / (rotary_dim - 2))
    i = torch.arange(0, rotary_dim, 2, dtype=torch.float64)
    f = base ** (-i / rotary_dim)
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "parts":
        if not fast_turns > slow_turns > 0:
            raise ValueError("parts scaling needs fast_turns > slow_turns > 0")
        # index at which a pair makes n turns over original_positions
        at = [rotary_dim / 2 * math.log(original_positions / (2 * math.pi * n)) / math.log(base)
              for n in (fast_turns, slow_turns)]
        # either end may lie outside the pairs there are: the line between them stays
        lo, hi = math.floor(at[0]), math.ceil(at[1])
        slow = ((i / 2 - lo) / max(hi - lo, 1)).clamp(0, 1)
        return f * (1 - slow) + f / factor * slow, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def ebd_rotary_table(inv_freq: torch.Tensor, n_pos: int, mscale: float = 1.0, table=None,
                     device=None, stream=None) -> torch.Tensor:
    """(cos, sin) of positions 0 .. n_pos - 1: float32 [n_pos, R / 2, 2] from the
    float64 frequencies [R / 2] (moved to `device` when they are on the CPU)."""
    if inv_freq.dtype != torch.float64 or inv_freq.dim() != 1:
        raise TypeError("inv_freq must be a one-dimensional float64 tensor")
    if table is None:
        dev = inv_freq.device if inv_freq.is_cuda else (device or "cuda")
        table = _result((n_pos, inv_freq.shape[0], 2), torch.float32, dev, stream)
    f = _on_device(inv_freq, table.device, stream)
    _check("ebd_rotary_table", lib().ebd_rotary_table(
        _ptr(f, name="inv_freq"), f.shape[0], int(n_pos), float(mscale),
        _ptr(table, torch.float32, (n_pos, f.shape[0], 2), "table"), _stream(stream)))
    return table


def ebd_rotary(x: torch.Tensor, positions: torch.Tensor, table: torch.Tensor, out=None,
               layout: int = EBD_ROTARY_HALF, inverse: bool = False, dev_status=None,
               stream=None) -> torch.Tensor:
    """x [T, H, d] (any token and head strides) turned to positions [T] (int32)
    with the table's rows; `inverse` turns back (the gradient).  out may be x."""
    if x.dim() != 3:
        raise ValueError("x must be [T, H, d]")
    T, H, d = x.shape
    if out is None:
        out = _result((T, H, d), x.dtype, x.device, stream)
    tab, n_pos, rot = _rotary_rows(table)
    xp, xt, xh = _rows(x, x.dtype, T, H, d, "x")
    yp, yt, yh = _rows(out, x.dtype, T, H, d, "out")
    _check("ebd_rotary", lib().ebd_rotary(
        _dtype_code(x), T, H, d, rot, int(layout), 1 if inverse else 0, xp, xt, xh,
        _ptr(positions, torch.int32, (T,), "positions"), tab, n_pos, yp, yt, yh,
        _ptr(dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return out


def ebd_paged_append(pc: PagedCache, k_new: torch.Tensor, v_new: torch.Tensor,
                     cu_new: torch.Tensor, table=None, layout: int = EBD_ROTARY_HALF, q=None,
                     q_out=None, stream=None) -> PagedCache:
    """Write the packed new tokens' keys (turned by the table, when given) and
    values into their pages; with q and q_out also the turned queries.
    k_new, v_new: [T, Hkv, d]; q, q_out: [T, Hq, d]; cu_new: [B + 1] int32."""
    c = _paged(pc)
    dt = pc.K_pages.dtype
    T, H, d = k_new.shape[0], c.n_kv_heads, c.head_dim
    kp, kt, kh = _rows(k_new, dt, T, H, d, "k_new")
    vp, vt, vh = _rows(v_new, dt, T, H, d, "v_new")
    tab, n_pos, rot = (None, 0, 0) if table is None else _rotary_rows(table)
    hq, qp, qt, qh, op, ot, oh = 0, None, 0, 0, None, 0, 0
    if q is not None:
        if q.dim() != 3 or q_out is None:
            raise ValueError("q must be [T, Hq, d] and come with q_out")
        hq = q.shape[1]
        qp, qt, qh = _rows(q, dt, T, hq, d, "q")
        op, ot, oh = _rows(q_out, dt, T, hq, d, "q_out")
    _check("ebd_paged_append", lib().ebd_paged_append(
        ctypes.byref(c), T, _ptr(cu_new, torch.int32, (c.batch + 1,), "cu_new"), kp, kt, kh, vp,
        vt, vh, tab, n_pos, rot, int(layout), hq, qp, qt, qh, op, ot, oh,
        _ptr(pc.dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return pc


def ebd_paged_attention_workspace_bytes(pc: PagedCache, n_q_heads: int, max_new: int) -> int:
    return int(lib().ebd_paged_attention_workspace_bytes(ctypes.byref(_paged(pc)), int(n_q_heads),
                                                         int(max_new)))


def ebd_paged_attention(q: torch.Tensor, pc: PagedCache, cu_new: torch.Tensor, max_new: int,
                        y=None, lse=None, scale=None, window: int = 0, workspace=None,
                        stream=None):
    """Causal attention of the packed new tokens q [T, Hq, d] over the paged
    cache that already holds their keys and values: y [T, Hq, d] in q's type and
    the log-sum-exp [T, Hq].  max_new: the most new tokens of any sequence;
    scale defaults to d^-1/2; window 0 sees every earlier position.  Tokens that cu_new
    gives to no sequence (EBD_DEV_RANGE in dev_status) keep what y and lse held."""
    if q.dim() != 3:
        raise ValueError("q must be [T, Hq, d]")
    c = _paged(pc)
    dt = pc.K_pages.dtype
    T, hq, d = q.shape[0], q.shape[1], c.head_dim
    qp, qt, qh = _rows(q, dt, T, hq, d, "q")
    if y is None:
        y = _result((T, hq, d), dt, q.device, stream)
    if lse is None:
        lse = _result((T, hq), torch.float32, q.device, stream)
    L = lib()
    ref = ctypes.byref(c)
    ws, wsb = _workspace(L.ebd_paged_attention_workspace_bytes(ref, hq, int(max_new)), q.device,
                         workspace, stream)
    _check("ebd_paged_attention", L.ebd_paged_attention(
        ref, T, int(max_new), hq, _ptr(cu_new, torch.int32, (c.batch + 1,), "cu_new"), qp, qt, qh,
        d ** -0.5 if scale is None else float(scale), int(window), _ptr(y, dt, (T, hq, d), "y"),
        _ptr(lse, torch.float32, (T, hq), "lse"),
        _ptr(pc.dev_status, torch.int32, (1,), "dev_status"), ws, wsb, _stream(stream)))
    return y, lse


def ebd_paged_gather(pc: PagedCache, out: CompactCache, stream=None) -> CompactCache:
    """Copy the cached rows named by out.idx_c into out.K_c / out.V_c."""
    c = _paged(pc)
    dt = pc.K_pages.dtype
    B, H, cap, d = c.batch, c.n_kv_heads, out.capacity, c.head_dim
    _check("ebd_paged_gather", lib().ebd_paged_gather(
        ctypes.byref(c), _ptr(out.idx_c, torch.int32, (B, H, cap), "idx_c"),
        _ptr(out.n_kept, torch.int32, (B, H), "n_kept"), cap,
        _ptr(out.K_c, dt, (B, H, cap, d), "K_c"), _ptr(out.V_c, dt, (B, H, cap, d), "V_c"),
        _ptr(out.dev_status, torch.int32, (1,), "dev_status"), _stream(stream)))
    return out


# ---------------------------------------------------------------- speculative steps
@dataclass
class PagePool:
    """The pages of a paged cache that nobody holds, and who holds which blocks.

    free_pages [n_pages] int32, of which the first n_free[0] are free; held [B, 2] int32:
    sequence b holds the pages of blocks held[b, 0] .. held[b, 1] - 1 of its row of the
    block table."""
    free_pages: torch.Tensor
    n_free: torch.Tensor
    held: torch.Tensor


def alloc_page_pool(batch, n_pages, device) -> PagePool:
    """Caller-side allocation: every page free, no sequence holds any."""
    i = torch.int32
    return PagePool(torch.arange(n_pages, dtype=i, device=device),
                    torch.full((1,), n_pages, dtype=i, device=device),
                    torch.zeros((batch, 2), dtype=i, device=device))


def ebd_paged_deal(pool: PagePool, pc: PagedCache, n_new: torch.Tensor, n_tokens: int,
                   window: int = 0, cu_new=None, positions=None, slots=None, served=None,
                   seq_len_out=None, held_out=None, n_free_out=None, stream=None):
    """Deal pages for n_new [B] (int32; negative: the sequence leaves) more tokens, at
    most n_tokens in all: (cu_new [B + 1], positions [n_tokens] int32, slots [n_tokens]
    int64, served [B]).  pc.seq_len counts the cached tokens before the call and, like
    pool.held and pool.n_free, is brought up to date in place unless another output is
    given; pc.block_table and pool.free_pages always are.  A sequence that is not served
    (EBD_DEV_CAPACITY in dev_status) has no new tokens in cu_new and keeps its length and
    pages, but for the blocks behind its window, which are given back like any other's
    (pool.held[b, 0] goes up; others may have been dealt their pages)."""
    B, i32, dev = pc.block_table.shape[0], torch.int32, pc.seq_len.device
    if cu_new is None:
        cu_new = _result((B + 1,), i32, dev, stream)
    if positions is None:
        positions = _result((n_tokens,), i32, dev, stream)
    if slots is None:
        slots = _result((n_tokens,), torch.int64, dev, stream)
    if served is None:
        served = _result((B,), i32, dev, stream)
    held, free, n = pool.held, pool.n_free, pc.seq_len
    _check("ebd_paged_deal", (_CALL or _call()).deal(
        pool.free_pages, free, held, pc.K_pages, pc.V_pages, pc.block_table, n, pc.dev_status,
        n_new, n_tokens, window, cu_new, positions, slots, served,
        n if seq_len_out is None else seq_len_out, held if held_out is None else held_out,
        free if n_free_out is None else n_free_out, stream))
    return cu_new, positions, slots, served


def ebd_norm_rotary(x: torch.Tensor, weight: torch.Tensor, positions=None, table=None, out=None,
                    layout: int = EBD_ROTARY_HALF, eps: float = 1e-6, dev_status=None,
                    stream=None) -> torch.Tensor:
    """x [T, H, d] (any token and head strides) divided by each row's root mean square,
    times weight ([d] or [H, d], x's type or float32), and, with a table, turned to
    positions [T] (int32).  out may be x."""
    if out is None:
        out = _result(x.shape, x.dtype, x.device, stream)
    _check("ebd_norm_rotary", (_CALL or _call()).norm(x, weight, positions, table, out, layout, eps,
                                                      dev_status, stream))
    return out


def ebd_norm_rotary_backward_workspace_bytes(n_heads: int, head_dim: int, per_head: bool) -> int:
    return int(lib().ebd_norm_rotary_backward_workspace_bytes(int(n_heads), int(head_dim),
                                                              1 if per_head else 0))


def ebd_norm_rotary_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor,
                             positions=None, table=None, dx=None, dweight=None,
                             layout: int = EBD_ROTARY_HALF, eps: float = 1e-6, workspace=None,
                             dev_status=None, stream=None):
    """Gradients of ebd_norm_rotary at x, given dy: dx [T, H, d] in x's type and dweight,
    float32 in the weight's shape.  dx may be dy or x."""
    if dx is None:
        dx = _result(x.shape, x.dtype, x.device, stream)
    if dweight is None:
        dweight = _result(weight.shape, torch.float32, x.device, stream)
    _check("ebd_norm_rotary_backward", (_CALL or _call()).norm_backward(
        dy, x, weight, positions, table, dx, dweight, layout, eps, workspace, dev_status, stream))
    return dx, dweight


def ebd_paged_append_norm(pc: PagedCache, k_new: torch.Tensor, v_new: torch.Tensor, k_weight=None,
                          q=None, q_weight=None, q_out=None, cu_new=None, slots=None,
                          positions=None, table=None, layout: int = EBD_ROTARY_HALF,
                          eps: float = 1e-6, stream=None) -> PagedCache:
    """ebd_paged_append with keys and queries normalised on the way (weights as for
    ebd_norm_rotary; None: not normalised), tokens placed by cu_new [B + 1] or by their
    slots [T] (int64, ebd_paged_deal; -1: no token).  positions [T]: where each is turned
    to; needed with slots and a table, otherwise a token's place in its sequence.  q_weight
    and q_out come with q."""
    _check("ebd_paged_append_norm", (_CALL or _call()).append_norm(
        pc.K_pages, pc.V_pages, pc.block_table, pc.seq_len, pc.dev_status, k_new, v_new, k_weight,
        q, q_weight, q_out, cu_new, slots, positions, table, layout, eps, stream))
    return pc


def ebd_tree_masks(parents: torch.Tensor, cu_new: torch.Tensor, seq_len: torch.Tensor,
                   max_new: int, window: int = 0, mask=None, positions=None, dev_status=None,
                   stream=None):
    """(mask [T, W] int32, positions [T] int32) of drafted trees from the parents [T] (int32)
    of their tokens: bit j of a token's row, W = ceil(max_new / 32) words, is set where it
    sees new token j of its sequence."""
    T, i32 = parents.shape[0], torch.int32
    if mask is None:
        mask = _result((T, -(-int(max_new) // 32)), i32, parents.device, stream)
    if positions is None:
        positions = _result((T,), i32, parents.device, stream)
    _check("ebd_tree_masks", (_CALL or _call()).tree_masks(
        parents, cu_new, seq_len, max_new, window, mask, positions, dev_status, stream))
    return mask, positions


def ebd_paged_tree_attention(q: torch.Tensor, pc: PagedCache, cu_new: torch.Tensor, max_new: int,
                             mask, positions=None, y=None, lse=None, scale=None,
                             window: int = 0, workspace=None, stream=None):
    """ebd_paged_attention of drafted trees: a new token sees the earlier positions and
    those new tokens of its sequence whose bits its row of mask [T, W] (int32,
    ebd_tree_masks) has; positions [T] are needed with a window.  mask None: no tree, every
    token sees those before it, as in ebd_paged_attention.  Places past the last offset (a
    deal's empty ones) are left alone."""
    if y is None:
        y = _result(q.shape, pc.K_pages.dtype, q.device, stream)
    if lse is None:
        lse = _result(q.shape[:2], torch.float32, q.device, stream)
    _check("ebd_paged_tree_attention", (_CALL or _call()).tree_attention(
        pc.K_pages, pc.V_pages, pc.block_table, pc.seq_len, pc.dev_status, q, cu_new, max_new,
        mask, positions, y, lse, scale, window, workspace, stream))
    return y, lse


def ebd_paged_keep(pc: PagedCache, cu_new: torch.Tensor, path: torch.Tensor,
                   n_accepted: torch.Tensor, seq_len_out=None, K_layers=None, V_layers=None,
                   stream=None) -> torch.Tensor:
    """Move the cached rows of each tree's accepted path (path [B, max_path] int32, rising
    numbers of new tokens; n_accepted [B]) to the places behind the tree's beginning,
    and return the new lengths [B].  K_layers, V_layers [L, n_pages, Hkv, page_size, d]:
    the pools of all layers, pc's among them as the first, moved in the same launch."""
    if seq_len_out is None:
        seq_len_out = _result(pc.seq_len.shape, torch.int32, pc.seq_len.device, stream)
    _check("ebd_paged_keep", (_CALL or _call()).keep(
        pc.K_pages, pc.V_pages, pc.block_table, pc.seq_len, pc.dev_status, cu_new, path, n_accepted,
        seq_len_out, K_layers, V_layers, stream))
    return seq_len_out
