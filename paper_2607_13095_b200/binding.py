"""Thin ctypes binding of libhswa.so: same names as the C ABI, argument marshalling only.

Tensors are torch CUDA tensors owned by the caller; this module passes their device pointers and the current
torch stream to the library.  Every step of the path runs inside the library's kernels; there is no Python or
CPU fallback, and a missing or unloadable library raises at import of the symbols.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional

import torch

from . import build as _build

HSWA_OK = 0
HSWA_ERR_INVALID_ARG = 1
HSWA_ERR_UNSUPPORTED = 2
HSWA_ERR_WORKSPACE = 3
HSWA_ERR_CUDA = 4
HSWA_ERR_BOUNDS = 5
HSWA_ERR_TIMEOUT = 6

EXPORTS = [
    "hswa_create", "hswa_destroy", "hswa_workspace_bytes", "hswa_validate_batch", "hswa_kv_append",
    "hswa_decode_attn", "hswa_decode_attn_mtp", "hswa_decode_attn_shared_prefix", "hswa_decode_attn_static_ws", "hswa_prefill_attn", "hswa_step_advance", "hswa_get_async_error", "hswa_status_string",
    "hswa_window_safe_len", "hswa_swa_window_gather", "hswa_swa_window_scatter",
    "hswa_decode_workspace_need", "hswa_selftest_wait_timeout", "hswa_set_overlap",
    "hswa_swa_release", "hswa_swa_valid_mask", "hswa_prefix_hit_len", "hswa_set_prefill_order", "hswa_set_block_trace",
    "hswa_probe_read_stream", "hswa_cross_attn", "hswa_cross_workspace_need", "hswa_attn_weights", "hswa_evict_select",
    "hswa_evict_compact", "hswa_packed_append", "hswa_packed_read", "hswa_packed_workspace_need", "hswa_packed_attn",
    "hswa_pages_workspace_need", "hswa_pages_fork", "hswa_pages_compact", "hswa_pages_copy",
]


class hswa_config(C.Structure):
    _fields_ = [
        ("num_q_heads", C.c_int32), ("num_kv_heads", C.c_int32), ("head_dim", C.c_int32),
        ("page_size", C.c_int32), ("window", C.c_int32), ("ring_pages", C.c_int32),
        ("sm_scale", C.c_float), ("out_dtype", C.c_int32),
    ]


class hswa_layer(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("num_pages", C.c_int64), ("is_swa", C.c_int32)]


class hswa_packed_layer(C.Structure):
    _fields_ = [("pool", C.c_void_p), ("num_pages", C.c_int64), ("k_scale", C.c_float), ("v_scale", C.c_float)]


class hswa_batch(C.Structure):
    _fields_ = [
        ("batch", C.c_int32), ("ctx_len", C.c_void_p), ("q_indptr", C.c_void_p), ("block_table", C.c_void_p),
        ("max_blocks", C.c_int32), ("ring_table", C.c_void_p), ("ring_head", C.c_void_p),
        ("max_q_len", C.c_int32), ("total_q", C.c_int32), ("max_ctx_len", C.c_int32),
    ]


class HswaError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


def _need(ok, what: str = "tensor of a wrong type, shape or size"):
    """A check of arguments; unlike an assert statement it stays under python -O, and the library trusts the sizes it passes."""
    if not ok:
        raise AssertionError(what)


_lib = None


def lib_path() -> str:
    return _build.LIB


def load(build_if_missing: bool = True) -> C.CDLL:
    """Load libhswa.so (building it in-tree first when it is absent or stale)."""
    global _lib
    if _lib is not None:
        return _lib
    path = _build.build() if build_if_missing else _build.LIB
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: run `python -m paper_2607_13095_b200.build`")
    lib = C.CDLL(path)
    vp, i32, i64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
    lib.hswa_create.restype = C.c_int
    lib.hswa_create.argtypes = [C.POINTER(hswa_config), C.POINTER(vp)]
    lib.hswa_destroy.restype = None
    lib.hswa_destroy.argtypes = [vp]
    lib.hswa_workspace_bytes.restype = sz
    lib.hswa_workspace_bytes.argtypes = [vp, i32, i32, i32]
    lib.hswa_decode_workspace_need.restype = sz
    lib.hswa_decode_workspace_need.argtypes = [vp, i32, i32, i32, i32, i32]
    lib.hswa_set_prefill_order.restype = C.c_int
    lib.hswa_set_prefill_order.argtypes = [vp, i32]
    lib.hswa_set_block_trace.restype = C.c_int
    lib.hswa_set_block_trace.argtypes = [vp, vp, i64]
    lib.hswa_probe_read_stream.restype = C.c_int
    lib.hswa_probe_read_stream.argtypes = [vp, vp, sz, vp]
    lib.hswa_set_overlap.restype = C.c_int
    lib.hswa_set_overlap.argtypes = [vp, i32]
    lib.hswa_selftest_wait_timeout.restype = C.c_int
    lib.hswa_selftest_wait_timeout.argtypes = [vp, i64, vp]
    lib.hswa_validate_batch.restype = C.c_int
    lib.hswa_validate_batch.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp]
    lib.hswa_kv_append.restype = C.c_int
    lib.hswa_kv_append.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, vp]
    lib.hswa_decode_attn.restype = C.c_int
    lib.hswa_decode_attn.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hswa_decode_attn_mtp.restype = C.c_int
    lib.hswa_decode_attn_mtp.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.hswa_decode_attn_shared_prefix.restype = C.c_int
    lib.hswa_decode_attn_shared_prefix.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), i32, vp, vp, vp, vp, vp,
                                                   vp, sz, vp]
    lib.hswa_decode_attn_static_ws.restype = C.c_int
    lib.hswa_decode_attn_static_ws.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, vp, vp, vp, vp]
    lib.hswa_prefill_attn.restype = C.c_int
    lib.hswa_prefill_attn.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, vp, i32, vp, vp, vp,
                                      sz, vp]
    lib.hswa_cross_workspace_need.restype = sz
    lib.hswa_cross_workspace_need.argtypes = [vp, i32, i32, i32, i32]
    lib.hswa_cross_attn.restype = C.c_int
    lib.hswa_cross_attn.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, vp, vp, sz, vp]
    lib.hswa_attn_weights.restype = C.c_int
    lib.hswa_attn_weights.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), i32, vp, vp, C.c_float, vp, i64, vp]
    lib.hswa_evict_select.restype = C.c_int
    lib.hswa_evict_select.argtypes = [vp, i32, vp, i32, vp, i64, vp, i32, i32, i32, vp, vp, vp]
    lib.hswa_evict_compact.restype = C.c_int
    lib.hswa_evict_compact.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp, i32, vp, i32, vp, i64, vp, i64, vp]
    for name in ("hswa_packed_append", "hswa_packed_read"):
        getattr(lib, name).restype = C.c_int
        getattr(lib, name).argtypes = [vp, C.POINTER(hswa_packed_layer), C.POINTER(hswa_batch), vp, vp, vp]
    lib.hswa_packed_workspace_need.restype = sz
    lib.hswa_packed_workspace_need.argtypes = [vp, i32, i32, i32, i32, i32]
    lib.hswa_packed_attn.restype = C.c_int
    lib.hswa_packed_attn.argtypes = [vp, C.POINTER(hswa_packed_layer), C.POINTER(hswa_batch), i32, vp, vp, vp, vp, sz, vp]
    lib.hswa_pages_workspace_need.restype = sz
    lib.hswa_pages_workspace_need.argtypes = [vp, i64]
    lib.hswa_pages_fork.restype = C.c_int
    lib.hswa_pages_fork.argtypes = [vp, i64, vp, vp, i32, vp, vp, i32, i32, vp, vp, vp, vp, i32, vp, vp, vp, vp, sz, vp]
    lib.hswa_pages_compact.restype = C.c_int
    lib.hswa_pages_compact.argtypes = [vp, i64, vp, vp, i32, vp, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.hswa_pages_copy.restype = C.c_int
    lib.hswa_pages_copy.argtypes = [vp, i32, C.POINTER(vp), i64, i64, i32, vp, vp, vp]
    lib.hswa_window_safe_len.restype = C.c_int64
    lib.hswa_window_safe_len.argtypes = [C.c_int64, i32, vp]
    lib.hswa_swa_window_gather.restype = C.c_int
    lib.hswa_swa_window_gather.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp]
    lib.hswa_swa_window_scatter.restype = C.c_int
    lib.hswa_swa_window_scatter.argtypes = [vp, C.POINTER(hswa_layer), C.POINTER(hswa_batch), vp, vp]
    lib.hswa_swa_release.restype = C.c_int
    lib.hswa_swa_release.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.hswa_swa_valid_mask.restype = C.c_int
    lib.hswa_swa_valid_mask.argtypes = [vp, i32, vp, vp, i64, vp, vp]
    lib.hswa_prefix_hit_len.restype = C.c_int64
    lib.hswa_prefix_hit_len.argtypes = [i64, i32, vp, vp]
    lib.hswa_step_advance.restype = C.c_int
    lib.hswa_step_advance.argtypes = [vp, i32, vp, vp, vp, vp]
    lib.hswa_get_async_error.restype = C.c_int
    lib.hswa_get_async_error.argtypes = [vp, vp, C.POINTER(i32 * 4)]
    lib.hswa_status_string.restype = C.c_char_p
    lib.hswa_status_string.argtypes = [C.c_int]
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().hswa_status_string(int(status)).decode()


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    _need(t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors")
    return t.data_ptr()


_device = torch._C._cuda_getDevice
_raw_stream = torch._C._cuda_getCurrentRawStream  # (without the Stream object around it: 0.2 us a call instead of 3.4 us)


def _stream():
    return _raw_stream(_device())


def _ptrs(dev: int, *tensors):
    """Addresses of contiguous tensors on CUDA device `dev` (None stays None)."""
    at = []
    for t in tensors:
        if t is None:
            at.append(None)
        elif t.get_device() != dev or not t.is_contiguous():
            raise AssertionError("device tensors must be contiguous CUDA tensors on the current device")
        else:
            at.append(t.data_ptr())
    return at


def _check(status: int, what: str):
    if status != HSWA_OK:
        raise HswaError(status, what)


class Handle:
    """Owns an hswa_handle*."""

    def __init__(self, num_q_heads, num_kv_heads, head_dim, page_size, window=128, ring_pages=0, sm_scale=0.0,
                 out_dtype=torch.bfloat16):
        self._h = C.c_void_p()
        self.cfg = hswa_config(num_q_heads, num_kv_heads, head_dim, page_size, window, ring_pages, sm_scale,
                               1 if out_dtype == torch.float32 else 0)
        self.out_dtype = out_dtype
        _check(load().hswa_create(C.byref(self.cfg), C.byref(self._h)), "hswa_create")
        self.packed_rows = (num_kv_heads, page_size * (head_dim // 2 + head_dim // 16))  # of a 4-bit pool: KV heads, bytes of a slab
        self.ring_pages = ring_pages or (-(-window // page_size) + 1)

    def close(self):
        if self._h:
            load().hswa_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def ptr(self):
        return self._h


def _pages_of(pool: torch.Tensor):
    """Where a pool's pages lie, their number and bytes."""
    n = int(pool.shape[0])
    return pool.data_ptr(), n, pool.numel() // n * pool.element_size() if n else 0


class Layer:
    """One layer's pool: bf16 CUDA tensor [num_pages][2][Hkv][P][D]."""

    def __init__(self, pool: torch.Tensor, is_swa: bool):
        _need(pool.dtype == torch.bfloat16 and pool.dim() == 5 and pool.is_contiguous())
        self.pool = pool
        self.device = pool.get_device()
        self.is_swa = bool(is_swa)
        self.pages = _pages_of(pool)
        self.c = hswa_layer(pool.data_ptr(), pool.shape[0], int(self.is_swa))
        self.ref = C.byref(self.c)


class PackedLayer:
    """A Full layer's 4-bit pool: uint8 CUDA tensor [num_pages][2][Hkv][P * (D / 2 + D / 16)] and the layer's scales of K and V."""

    def __init__(self, pool: torch.Tensor, k_scale: float = 1.0, v_scale: float = 1.0):
        _need(pool.dtype == torch.uint8 and pool.dim() == 4 and pool.shape[1] == 2 and pool.is_contiguous())
        self.pool = pool
        self.device = pool.get_device()
        self.rows = tuple(pool.shape[2:])  # KV heads, bytes of a slab
        self.pages = _pages_of(pool)
        self.c = hswa_packed_layer(pool.data_ptr(), pool.shape[0], k_scale, v_scale)
        self.ref = C.byref(self.c)


class Batch:
    """One step's batch: int32 CUDA tensors plus the host-known bounds."""

    def __init__(self, ctx_len, block_table, ring_table, ring_head, q_indptr=None, *, max_q_len=1, total_q=None,
                 max_ctx_len=0):
        for t in (ctx_len, block_table, ring_table, ring_head):
            _need(t.dtype == torch.int32 and t.is_cuda and t.is_contiguous())
        self.ctx_len, self.block_table, self.ring_table, self.ring_head, self.q_indptr = (
            ctx_len, block_table, ring_table, ring_head, q_indptr)
        B = int(ctx_len.shape[0])
        self.batch = B
        self.device = ctx_len.get_device()
        # (what the calls on Full layers' contexts ask of the arrays besides their types)
        self.covers_batch = block_table.dim() == 2 and block_table.shape[0] >= B and (
            q_indptr is None or (q_indptr.dtype == torch.int32 and q_indptr.is_cuda and q_indptr.is_contiguous() and q_indptr.numel() > B))
        self.total_q = B if total_q is None else int(total_q)
        self.max_q_len = int(max_q_len)
        self.c = hswa_batch(
            B, ctx_len.data_ptr(), None if q_indptr is None else q_indptr.data_ptr(), block_table.data_ptr(),
            int(block_table.shape[1]) if block_table.dim() == 2 else 0, ring_table.data_ptr(), ring_head.data_ptr(),
            self.max_q_len, self.total_q, int(max_ctx_len))
        self.ref = C.byref(self.c)


def hswa_workspace_bytes(h: Handle, max_batch: int, max_total_q: int, max_ctx_len: int) -> int:
    return int(load().hswa_workspace_bytes(h.ptr, max_batch, max_total_q, max_ctx_len))


def hswa_decode_workspace_need(h: Handle, is_swa: bool, batch: int, max_ctx_len: int, shared_prefix_len: int = 0,
                               q_len: int = 1) -> int:
    return int(load().hswa_decode_workspace_need(h.ptr, int(bool(is_swa)), batch, max_ctx_len, shared_prefix_len, q_len))


def hswa_set_overlap(h: Handle, enabled: bool):
    _check(load().hswa_set_overlap(h.ptr, int(bool(enabled))), "hswa_set_overlap")


PREFILL_ORDER_BY_REQUEST, PREFILL_ORDER_LAST_TILE_FIRST, PREFILL_ORDER_LONGEST_REQUEST_FIRST, PREFILL_ORDER_LONGEST_TILE_FIRST = 0, 1, 2, 3


def hswa_set_prefill_order(h: Handle, mode: int):
    _check(load().hswa_set_prefill_order(h.ptr, int(mode)), "hswa_set_prefill_order")


def hswa_set_block_trace(h: Handle, buf: Optional[torch.Tensor]):
    """buf: int64 CUDA tensor [capacity][4] (zeroed by the caller) or None to switch the trace off."""
    if buf is None:
        _check(load().hswa_set_block_trace(h.ptr, None, 0), "hswa_set_block_trace")
        return
    _need(buf.dtype == torch.int64 and buf.is_cuda and buf.is_contiguous() and buf.dim() == 2 and buf.shape[1] == 4)
    _check(load().hswa_set_block_trace(h.ptr, C.c_void_p(buf.data_ptr()), int(buf.shape[0])), "hswa_set_block_trace")


def hswa_probe_read_stream(h: Handle, buf: torch.Tensor):
    """Stream a CUDA tensor's bytes (a multiple of 32 KB) through shared memory; time it with events."""
    _check(load().hswa_probe_read_stream(h.ptr, _ptr(buf), buf.numel() * buf.element_size(), _stream()), "hswa_probe_read_stream")


def hswa_selftest_wait_timeout(h: Handle, limit_clocks: int):
    _check(load().hswa_selftest_wait_timeout(h.ptr, int(limit_clocks), _stream()), "hswa_selftest_wait_timeout")


def hswa_validate_batch(h: Handle, layer: Layer, batch: Batch):
    _check(load().hswa_validate_batch(h.ptr, C.byref(layer.c), C.byref(batch.c), _stream()), "hswa_validate_batch")


def hswa_kv_append(h: Handle, layer: Layer, batch: Batch, k_new: torch.Tensor, v_new: torch.Tensor):
    _check(load().hswa_kv_append(h.ptr, C.byref(layer.c), C.byref(batch.c), _ptr(k_new), _ptr(v_new), _stream()),
           "hswa_kv_append")


def hswa_decode_attn(h: Handle, layer: Layer, batch: Batch, q, k_new, v_new, out, lse=None, workspace=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().hswa_decode_attn(h.ptr, C.byref(layer.c), C.byref(batch.c), _ptr(q), _ptr(k_new), _ptr(v_new),
                                   _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream()), "hswa_decode_attn")


def hswa_decode_attn_mtp(h: Handle, layer: Layer, batch: Batch, q_len: int, q, k_new, v_new, out, lse=None, workspace=None):
    """Multi-token decode: q [B][q_len][Hq][D], k_new / v_new [B][q_len][Hkv][D], causal within the q_len drafts."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().hswa_decode_attn_mtp(h.ptr, C.byref(layer.c), C.byref(batch.c), int(q_len), _ptr(q), _ptr(k_new),
                                       _ptr(v_new), _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes, _stream()),
           "hswa_decode_attn_mtp")


def hswa_decode_attn_shared_prefix(h: Handle, layer: Layer, batch: Batch, shared_prefix_len: int, q, k_new, v_new, out,
                                   lse=None, workspace=None):
    """Cascade decode: every request of the batch shares its first shared_prefix_len cached tokens (same pages)."""
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().hswa_decode_attn_shared_prefix(h.ptr, C.byref(layer.c), C.byref(batch.c), int(shared_prefix_len), _ptr(q),
                                                 _ptr(k_new), _ptr(v_new), _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes,
                                                 _stream()), "hswa_decode_attn_shared_prefix")


STATIC_WS_BYTES = 64 << 20


def hswa_decode_attn_static_ws(h: Handle, layer: Layer, batch: Batch, q, k_new, v_new, out, lse=None):
    """Decode attention for callers that cannot allocate: the split-K scratch is a fixed STATIC_WS_BYTES array
    inside the library (shared by all calls on the device, so keep them on one stream).  Make the first call
    on a device outside any stream capture."""
    _check(load().hswa_decode_attn_static_ws(h.ptr, C.byref(layer.c), C.byref(batch.c), _ptr(q), _ptr(k_new),
                                             _ptr(v_new), _ptr(out), _ptr(lse), _stream()),
           "hswa_decode_attn_static_ws")


def hswa_prefill_attn(h: Handle, layer: Layer, batch: Batch, q, k_new, v_new, fuse_append, out, lse=None,
                      workspace=None):
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load().hswa_prefill_attn(h.ptr, C.byref(layer.c), C.byref(batch.c), _ptr(q), _ptr(k_new), _ptr(v_new),
                                    int(bool(fuse_append)), _ptr(out), _ptr(lse), _ptr(workspace), ws_bytes,
                                    _stream()), "hswa_prefill_attn")


def hswa_cross_workspace_need(h: Handle, batch: int, total_q: int, max_q_len: int, max_ctx_len: int) -> int:
    return int(load().hswa_cross_workspace_need(h.ptr, batch, total_q, max_q_len, max_ctx_len))


def _device_of(layer, batch: Batch) -> int:
    """The current device, which has to be that of the layer and the batch."""
    if not batch.covers_batch:
        raise AssertionError("block_table needs a row per request and q_indptr, int32, one entry more")
    dev = _device()
    if not layer.device == batch.device == dev:
        raise AssertionError("layer or batch on another device than the current one")
    return dev


def _rows_are_said(batch: Batch, q):
    # [B][q_len][Hq][D], as multi-token decode takes it: without row offsets its r-th row would count as request r's
    _need(batch.q_indptr is not None or q.dim() < 4 or q.shape[1] == 1, "several rows of q per request need q_indptr")


def hswa_cross_attn(h: Handle, layer: Layer, batch: Batch, q, out, lse=None, workspace=None):
    """Attention of q [T][Hq][D] to all ctx_len[r] cached states of each request (no causal mask, nothing appended)."""
    _need(q.dtype == torch.bfloat16 and out.dtype == h.out_dtype and (lse is None or lse.dtype == torch.float32))
    _rows_are_said(batch, q)
    rows = batch.total_q * h.cfg.num_q_heads
    n = rows * h.cfg.head_dim
    _need(q.numel() >= n and out.numel() >= n and (lse is None or lse.numel() >= rows), "fewer rows than total_q")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    dev = _device_of(layer, batch)
    _check(load().hswa_cross_attn(h.ptr, layer.ref, batch.ref, *_ptrs(dev, q, out, lse, workspace), ws_bytes, _raw_stream(dev)),
           "hswa_cross_attn")


def hswa_attn_weights(h: Handle, layer: Layer, batch: Batch, causal: bool, q, lse, decay: float, weights: torch.Tensor):
    """weights: fp32 CUDA tensor [B][Hkv][stride], updated in place with the attention weights of q's rows (lse: theirs).

    After hswa_decode_attn_mtp: a Batch with q_indptr = arange(B + 1) * q_len; an lse of -inf takes a draft's vote away."""
    _need(q.dtype == torch.bfloat16 and lse.dtype == torch.float32)
    _rows_are_said(batch, q)
    B, heads, stride = weights.shape
    _need(weights.dtype == torch.float32 and B == batch.batch and heads == h.cfg.num_kv_heads)
    rows = batch.total_q * h.cfg.num_q_heads
    _need(q.numel() >= rows * h.cfg.head_dim and lse.numel() >= rows, "fewer rows than total_q")
    dev = _device_of(layer, batch)
    q_at, lse_at, weights_at = _ptrs(dev, q, lse, weights)
    _check(load().hswa_attn_weights(h.ptr, layer.ref, batch.ref, bool(causal), q_at, lse_at, decay, weights_at, stride,
                                    _raw_stream(dev)), "hswa_attn_weights")


def hswa_evict_select(h: Handle, batch: int, ctx_len: torch.Tensor, max_ctx_len: int, weights: torch.Tensor, keep_len: torch.Tensor,
                      keep_idx: torch.Tensor, kept_len: torch.Tensor, *, protect_first: int = 0, protect_last: int = 0):
    """keep_idx: int32 CUDA tensor [B][Hkv][max_keep], filled with the positions of largest weight, ascending, then -1."""
    i32, heads = torch.int32, h.cfg.num_kv_heads
    _need(ctx_len.dtype == i32 and keep_len.dtype == i32 and keep_idx.dtype == i32 and kept_len.dtype == i32)
    w_batch, w_heads, stride = weights.shape
    k_batch, k_heads, max_keep = keep_idx.shape
    _need(weights.dtype == torch.float32 and w_batch == k_batch == batch and w_heads == k_heads == heads)
    _need(ctx_len.numel() >= batch and keep_len.numel() >= batch and kept_len.numel() >= batch)
    dev = _device()
    ctx_at, weights_at, keep_at, idx_at, kept_at = _ptrs(dev, ctx_len, weights, keep_len, keep_idx, kept_len)
    _check(load().hswa_evict_select(h.ptr, batch, ctx_at, max_ctx_len, weights_at, stride, keep_at, max_keep, protect_first,
                                    protect_last, idx_at, kept_at, _raw_stream(dev)), "hswa_evict_select")


def hswa_evict_compact(h: Handle, layer: Layer, batch: Batch, keep_idx: torch.Tensor, kept_len: torch.Tensor,
                       dst_block_table: torch.Tensor, weights: Optional[torch.Tensor] = None,
                       weights_out: Optional[torch.Tensor] = None):
    """Copies the kept K/V rows (and weights) of batch's block table to the pages of dst_block_table [B][blocks]."""
    i32, f32 = torch.int32, torch.float32
    _need(keep_idx.dtype == i32 and kept_len.dtype == i32 and dst_block_table.dtype == i32)
    _need((weights is None or weights.dtype == f32) and (weights_out is None or weights_out.dtype == f32))
    B, heads, max_keep = keep_idx.shape
    dst_batch, dst_blocks = dst_block_table.shape
    _need(B == dst_batch == batch.batch and heads == h.cfg.num_kv_heads and kept_len.numel() >= B)
    stride = out_stride = 0
    if weights is not None:
        w_batch, w_heads, stride = weights.shape
        _need(w_batch == B and w_heads == heads)
    if weights_out is not None:
        w_batch, w_heads, out_stride = weights_out.shape
        _need(w_batch == B and w_heads == heads)
    dev = _device_of(layer, batch)
    idx_at, kept_at, dst_at, weights_at, out_at = _ptrs(dev, keep_idx, kept_len, dst_block_table, weights, weights_out)
    _check(load().hswa_evict_compact(h.ptr, layer.ref, batch.ref, idx_at, kept_at, max_keep, dst_at, dst_blocks, weights_at, stride,
                                     out_at, out_stride, _raw_stream(dev)), "hswa_evict_compact")


def _packed_device_of(h: Handle, layer: PackedLayer, batch: Batch) -> int:
    _need(layer.rows == h.packed_rows, "4-bit pool of another head count, head dim or page size than the handle's")
    return _device_of(layer, batch)


def _packed_rows(call, what, h: Handle, layer: PackedLayer, batch: Batch, k: torch.Tensor, v: torch.Tensor):
    n = batch.total_q * h.packed_rows[0] * h.cfg.head_dim
    _need(k.dtype == v.dtype == torch.bfloat16 and k.numel() >= n and v.numel() >= n, "k and v: bf16, total_q rows")
    dev = _packed_device_of(h, layer, batch)
    k_at, v_at = _ptrs(dev, k, v)
    _check(call(h.ptr, layer.ref, batch.ref, k_at, v_at, _raw_stream(dev)), what)


_is_contiguous, _get_device, _data_ptr, _INT32 = torch.Tensor.is_contiguous, torch.Tensor.get_device, torch.Tensor.data_ptr, {torch.int32}


def _int_ptrs(dev: int, *tensors):
    """_ptrs of int32 tensors."""
    if not (all(map(_is_contiguous, tensors)) and set(map(_get_device, tensors)) == {dev} and {t.dtype for t in tensors} == _INT32):
        raise AssertionError("device tensors must be contiguous int32 CUDA tensors on the current device")
    return map(_data_ptr, tensors)


def hswa_packed_append(h: Handle, layer: PackedLayer, batch: Batch, k_new: torch.Tensor, v_new: torch.Tensor):
    """Rounds k_new, v_new [T][Hkv][D] to 4 bits at the positions from ctx_len[r] on."""
    _packed_rows(load().hswa_packed_append, "hswa_packed_append", h, layer, batch, k_new, v_new)


def hswa_packed_read(h: Handle, layer: PackedLayer, batch: Batch, k_out: torch.Tensor, v_out: torch.Tensor):
    """The rows at the positions from ctx_len[r] on, as bf16 [T][Hkv][D]."""
    _packed_rows(load().hswa_packed_read, "hswa_packed_read", h, layer, batch, k_out, v_out)


def hswa_packed_workspace_need(h: Handle, batch: int, total_q: int, max_q_len: int, max_ctx_len: int, causal: bool) -> int:
    return int(load().hswa_packed_workspace_need(h.ptr, batch, total_q, max_q_len, max_ctx_len, bool(causal)))


def hswa_packed_attn(h: Handle, layer: PackedLayer, batch: Batch, causal: bool, q, out, lse=None, workspace=None):
    """Attention of q [T][Hq][D] over a 4-bit cache: causal (the step's rows appended before), or to all ctx_len[r] positions."""
    _need(q.dtype == torch.bfloat16 and out.dtype == h.out_dtype and (lse is None or lse.dtype == torch.float32))
    _rows_are_said(batch, q)
    rows = batch.total_q * h.cfg.num_q_heads
    n = rows * h.cfg.head_dim
    _need(q.numel() >= n and out.numel() >= n and (lse is None or lse.numel() >= rows), "fewer rows than total_q")
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    dev = _packed_device_of(h, layer, batch)
    q_at, out_at, lse_at, ws_at = _ptrs(dev, q, out, lse, workspace)
    _check(load().hswa_packed_attn(h.ptr, layer.ref, batch.ref, bool(causal), q_at, out_at, lse_at, ws_at, ws_bytes, _raw_stream(dev)),
           "hswa_packed_attn")


def hswa_pages_workspace_need(h: Handle, num_pages: int) -> int:
    return int(load().hswa_pages_workspace_need(h.ptr, num_pages))


def hswa_pages_fork(h: Handle, ref, ref_out, table, held, parent, length, need, table_out, held_out, copy_src, copy_dst, workspace):
    """Block tables of a step's rows from their parents': int32 CUDA tensors, ref [num_pages], table [rows][blocks], the others [rows]."""
    rows_in, blocks = table.shape
    rows_out, out_blocks = table_out.shape
    pages = ref.numel()
    _need(ref_out.numel() == pages)
    _need(held.numel() >= rows_in and min(parent.numel(), length.numel(), need.numel(), held_out.numel(), copy_src.numel(), copy_dst.numel()) >= rows_out,
          "fewer entries than rows")
    dev = _device()
    ref_at, ref_out_at, held_at, table_at, parent_at, len_at, need_at, table_out_at, held_out_at, src_at, dst_at = _int_ptrs(
        dev, ref, ref_out, held, table, parent, length, need, table_out, held_out, copy_src, copy_dst)
    ws_at, = _ptrs(dev, workspace)
    _check(load().hswa_pages_fork(h.ptr, pages, ref_at, ref_out_at, rows_in, held_at, table_at, blocks, rows_out, parent_at, len_at, need_at,
                                  table_out_at, out_blocks, held_out_at, src_at, dst_at, ws_at, workspace.numel() * workspace.element_size(),
                                  _raw_stream(dev)), "hswa_pages_fork")


def hswa_pages_compact(h: Handle, ref, ref_out, table, held, table_out, page_map, move_src, move_dst):
    """Moves of live pages into the lowest free ones, as many as move_src has places: int32 CUDA tensors."""
    rows, blocks = table.shape
    pages, moves = ref.numel(), move_src.numel()
    _need(ref_out.numel() == page_map.numel() == pages and table_out.shape == table.shape and held.numel() >= rows and move_dst.numel() == moves)
    dev = _device()
    ref_at, ref_out_at, held_at, table_at, table_out_at, map_at, src_at, dst_at = _int_ptrs(
        dev, ref, ref_out, held, table, table_out, page_map, move_src, move_dst)
    _check(load().hswa_pages_compact(h.ptr, pages, ref_at, ref_out_at, rows, held_at, table_at, blocks, table_out_at, map_at, moves, src_at,
                                     dst_at, _raw_stream(dev)), "hswa_pages_compact")


def hswa_pages_copy(h: Handle, layers, src: torch.Tensor, dst: torch.Tensor):
    """layers: Layer or PackedLayer objects of one kind and size, any number of them; pairs of page ids, -1 where there is none."""
    pairs = src.numel()
    _need(src.dtype == dst.dtype == torch.int32 and dst.numel() == pairs)
    if not layers:
        return
    dev = _device()
    _, num_pages, page_bytes = layers[0].pages
    pools = (C.c_void_p * len(layers))()
    for i, x in enumerate(layers):
        pools[i], n, size = x.pages
        if n != num_pages or size != page_bytes:
            raise AssertionError("pools of different sizes")
        if x.device != dev:
            raise AssertionError("layer on another device than the current one")
    src_at, dst_at = _ptrs(dev, src, dst)
    _check(load().hswa_pages_copy(h.ptr, len(layers), pools, num_pages, page_bytes, pairs, src_at, dst_at, _raw_stream(dev)), "hswa_pages_copy")


def hswa_window_safe_len(match_len: int, window: int, swa_valid) -> int:
    """Largest usable hit length given the donor's per-position SWA validity (any uint8 buffer / numpy array)."""
    import numpy as np
    v = np.ascontiguousarray(swa_valid, dtype=np.uint8)
    _need(v.shape[0] >= match_len)
    return int(load().hswa_window_safe_len(int(match_len), int(window), C.c_void_p(v.ctypes.data)))


def _any_ptr(t: torch.Tensor):
    _need(t.is_contiguous() and (t.is_cuda or t.is_pinned()), "buffer must be a CUDA tensor or pinned host memory")
    return C.c_void_p(t.data_ptr())


def hswa_swa_window_gather(h: Handle, layer: Layer, batch: Batch, buf: torch.Tensor):
    _check(load().hswa_swa_window_gather(h.ptr, C.byref(layer.c), C.byref(batch.c), _any_ptr(buf), _stream()),
           "hswa_swa_window_gather")


def hswa_swa_window_scatter(h: Handle, layer: Layer, batch: Batch, buf: torch.Tensor):
    _check(load().hswa_swa_window_scatter(h.ptr, C.byref(layer.c), C.byref(batch.c), _any_ptr(buf), _stream()),
           "hswa_swa_window_scatter")


def hswa_swa_release(h: Handle, batch: int, ctx_len: torch.Tensor, release: Optional[torch.Tensor],
                     swa_valid_from: torch.Tensor):
    """release: uint8 CUDA tensor [B] (None: every request releases); swa_valid_from: int32 CUDA tensor [B], in place."""
    _need(swa_valid_from.dtype == torch.int32 and (release is None or release.dtype == torch.uint8))
    _check(load().hswa_swa_release(h.ptr, batch, _ptr(ctx_len), _ptr(release), _ptr(swa_valid_from), _stream()),
           "hswa_swa_release")


def hswa_swa_valid_mask(h: Handle, batch: int, ctx_len: torch.Tensor, swa_valid_from: torch.Tensor, mask: torch.Tensor):
    """mask: uint8 [B][stride], CUDA or pinned host."""
    _need(mask.dtype == torch.uint8 and mask.dim() == 2 and mask.shape[0] == batch)
    _check(load().hswa_swa_valid_mask(h.ptr, batch, _ptr(ctx_len), _ptr(swa_valid_from), int(mask.shape[1]), _any_ptr(mask),
                                      _stream()), "hswa_swa_valid_mask")


def hswa_prefix_hit_len(match_len: int, window: int, full_valid, swa_valid) -> int:
    import numpy as np
    f = np.ascontiguousarray(full_valid, dtype=np.uint8)
    s = np.ascontiguousarray(swa_valid, dtype=np.uint8)
    _need(f.shape[0] >= match_len and s.shape[0] >= match_len)
    return int(load().hswa_prefix_hit_len(int(match_len), int(window), C.c_void_p(f.ctypes.data), C.c_void_p(s.ctypes.data)))


def hswa_step_advance(h: Handle, batch: int, ctx_len: torch.Tensor, ring_head: torch.Tensor, q_indptr=None):
    _check(load().hswa_step_advance(h.ptr, batch, _ptr(ctx_len), _ptr(ring_head), _ptr(q_indptr), _stream()),
           "hswa_step_advance")


def hswa_get_async_error(h: Handle):
    """Synchronise the current stream and return (status, request, index, value); clears the error word."""
    info = (C.c_int32 * 4)()
    st = load().hswa_get_async_error(h.ptr, _stream(), C.byref(info))
    return int(st), int(info[1]), int(info[2]), int(info[3])
