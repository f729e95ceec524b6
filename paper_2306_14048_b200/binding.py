"""ctypes binding of libh2o_b200.so: the same calls as include/h2o.h, argument marshalling only.

Every step of the path runs in the CUDA kernels behind the C ABI.  PyTorch is
used here for device memory and streams, nothing else.  There is no fallback:
if the shared library is missing the import of this module fails; if the
_pages extension for this Python and torch is, H2ORotary and H2OPages do.
"""
from __future__ import annotations

import ctypes
import importlib.util
import os
import struct
from typing import Optional, Sequence

import numpy as np
import torch

from .build import pages_path

_PKG = os.path.dirname(os.path.abspath(__file__))
# H2O_B200_LIB names another build of the same library (the checked variant libh2o_b200_bounds.so of build.py)
LIB_PATH = os.environ.get("H2O_B200_LIB") or os.path.join(_PKG, "libh2o_b200.so")

H2O_OK = 0
H2O_ERR_INVALID_ARG = -1
H2O_ERR_UNSUPPORTED = -2
H2O_ERR_WORKSPACE = -3
H2O_ERR_STATE = -4
H2O_ERR_CUDA = -5
H2O_ERR_TIMEOUT = -6
H2O_F32 = 0
H2O_BF16 = 1
H2O_BF16_KV4 = 2  # bf16 inputs, 4-bit group-quantised K/V slots
H2O_KV8 = 3  # rows of an H2OStore as e4m3 codes and one power of two per row and head

EXPORTED = (
    "h2o_cache_workspace_bytes",
    "h2o_prefill_scratch_bytes",
    "h2o_cache_create",
    "h2o_prefill_select",
    "h2o_prefill_select_static",
    "h2o_prefill_static_scratch_bytes",
    "h2o_decode_step",
    "h2o_cache_destroy",
    "h2o_cache_reset",
    "h2o_host_staging_bytes",
    "h2o_prefill_select_host",
    "h2o_decode_step_host",
    "h2o_cache_export",
    "h2o_cache_status",
    "h2o_cache_set_decode_shape",
    "h2o_cache_set_prefill_path",
    "h2o_cache_set_decode_path",
    "h2o_cache_get_decode_path",
    "h2o_debug_set_early_prefetch",
    "h2o_prefill_scratch_layout",
    "h2o_store_create",
    "h2o_store_destroy",
    "h2o_debug_store_set_polls",
    "h2o_store_write",
    "h2o_store_read",
    "h2o_cross_scratch_bytes",
    "h2o_cross_attend",
    "h2o_prefix_scratch_bytes",
    "h2o_prefix_attend",
    "h2o_rotate",
    "h2o_pages_create",
    "h2o_pages_destroy",
    "h2o_debug_pages_set_polls",
    "h2o_pages_append",
    "h2o_pages_scratch_bytes",
    "h2o_pages_attend",
    "h2o_strerror",
)


class h2o_config_t(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32),
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("heavy_budget", ctypes.POINTER(ctypes.c_int32)),
        ("recent_window", ctypes.POINTER(ctypes.c_int32)),
        ("softmax_scale", ctypes.c_float),
        ("device", ctypes.c_int32),
        ("query_group", ctypes.c_int32),
    ]


class h2o_store_config_t(ctypes.Structure):
    _fields_ = [
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("format", ctypes.c_int32),
        ("device", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("row_stride", ctypes.c_int64),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("k_scale", ctypes.c_void_p),
        ("v_scale", ctypes.c_void_p),
        ("status", ctypes.c_void_p),
    ]


class h2o_queries_t(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p),
        ("out", ctypes.c_void_p),
        ("lse", ctypes.c_void_p),
        ("cu_q", ctypes.c_void_p),
        ("q_rows", ctypes.c_int64),
        ("q_stride", ctypes.c_int64),
        ("out_stride", ctypes.c_int64),
        ("softmax_scale", ctypes.c_float),
        ("dtype", ctypes.c_int32),
        ("query_group", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("max_q", ctypes.c_int32),
    ]


class h2o_ranges_t(ctypes.Structure):
    _fields_ = [("begin", ctypes.c_void_p), ("length", ctypes.c_void_p), ("max_length", ctypes.c_int32)]


class h2o_rotary_t(ctypes.Structure):
    _fields_ = [
        ("frequency", ctypes.c_void_p),
        ("axis", ctypes.c_void_p),
        ("rotary_dim", ctypes.c_int32),
        ("axes", ctypes.c_int32),
        ("pairs", ctypes.c_int32),
        ("device", ctypes.c_int32),
        ("status", ctypes.c_void_p),
    ]


class h2o_pages_config_t(ctypes.Structure):
    _fields_ = [
        ("n_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("format", ctypes.c_int32),
        ("device", ctypes.c_int32),
        ("n_pages", ctypes.c_int32),
        ("page_size", ctypes.c_int32),
        ("page_stride", ctypes.c_int64),
        ("row_stride", ctypes.c_int64),
        ("head_stride", ctypes.c_int64),
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("status", ctypes.c_void_p),
    ]


class h2o_sequences_t(ctypes.Structure):
    _fields_ = [
        ("table", ctypes.c_void_p),
        ("length", ctypes.c_void_p),
        ("table_stride", ctypes.c_int64),
        ("max_pages", ctypes.c_int32),
        ("max_length", ctypes.c_int32),
    ]


class h2o_tokens_t(ctypes.Structure):
    _fields_ = [
        ("k", ctypes.c_void_p),
        ("v", ctypes.c_void_p),
        ("q", ctypes.c_void_p),
        ("q_out", ctypes.c_void_p),
        ("cu", ctypes.c_void_p),
        ("positions", ctypes.c_void_p),
        ("n_tokens", ctypes.c_int64),
        ("kv_stride", ctypes.c_int64),
        ("q_stride", ctypes.c_int64),
        ("q_out_stride", ctypes.c_int64),
        ("position_stride", ctypes.c_int64),
        ("query_group", ctypes.c_int32),
        ("batch", ctypes.c_int32),
    ]


def _load() -> ctypes.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libh2o_b200.so is not built (run `python paper_2306_14048_b200/build.py`); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    c = ctypes
    vp, i32p = c.c_void_p, c.POINTER(c.c_int32)
    cfgp = c.POINTER(h2o_config_t)
    lib.h2o_cache_workspace_bytes.restype = c.c_size_t
    lib.h2o_cache_workspace_bytes.argtypes = [cfgp]
    lib.h2o_prefill_scratch_bytes.restype = c.c_size_t
    lib.h2o_prefill_scratch_bytes.argtypes = [cfgp, c.c_int64]
    lib.h2o_cache_create.restype = c.c_int
    lib.h2o_cache_create.argtypes = [c.POINTER(vp), cfgp, vp, c.c_size_t]
    lib.h2o_prefill_select.restype = c.c_int
    lib.h2o_debug_wait_probe.argtypes = [vp, c.c_int32, vp]
    lib.h2o_debug_wait_probe.restype = c.c_int
    lib.h2o_cache_attach.argtypes = [c.POINTER(vp), cfgp, vp, c.c_size_t]
    lib.h2o_cache_attach.restype = c.c_int
    lib.h2o_prefill_select.argtypes = [vp, vp, vp, vp, i32p, vp, vp, c.c_size_t, vp]
    lib.h2o_prefill_select_static.restype = c.c_int
    lib.h2o_prefill_select_static.argtypes = [vp, vp, vp, vp, i32p, vp, vp]
    lib.h2o_prefill_static_scratch_bytes.restype = c.c_size_t
    lib.h2o_prefill_static_scratch_bytes.argtypes = []
    lib.h2o_decode_step.restype = c.c_int
    lib.h2o_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp]
    lib.h2o_cache_reset.restype = c.c_int
    lib.h2o_decode_chunk.argtypes = [vp, vp, vp, vp, c.c_int32, vp, vp, vp]
    lib.h2o_decode_chunk.restype = c.c_int
    lib.h2o_cache_set_chunk_path.argtypes = [vp, c.c_int32]
    lib.h2o_cache_set_chunk_path.restype = c.c_int
    lib.h2o_cache_set_score_mode.argtypes = [vp, c.c_int32]
    lib.h2o_cache_set_score_mode.restype = c.c_int
    lib.h2o_cache_set_topk.argtypes = [vp, c.c_int32]
    lib.h2o_cache_set_topk.restype = c.c_int
    lib.h2o_cache_set_mask.argtypes = [vp, c.c_int32, c.c_int32, c.c_int32]
    lib.h2o_cache_set_mask.restype = c.c_int
    lib.h2o_cache_fscore.argtypes = [vp, c.c_int32, vp, vp]
    lib.h2o_cache_fscore.restype = c.c_int
    lib.h2o_cache_reset.argtypes = [vp, vp]
    lib.h2o_host_staging_bytes.restype = c.c_size_t
    lib.h2o_host_staging_bytes.argtypes = [cfgp, c.c_int64]
    lib.h2o_prefill_select_host.restype = c.c_int
    lib.h2o_prefill_select_host.argtypes = [vp, vp, vp, vp, i32p, vp, vp, c.c_size_t, vp, c.c_size_t, vp]
    lib.h2o_decode_step_host.restype = c.c_int
    lib.h2o_decode_step_host.argtypes = [vp, vp, vp, vp, vp, vp, vp, c.c_size_t, vp]
    lib.h2o_cache_destroy.restype = c.c_int
    lib.h2o_cache_destroy.argtypes = [vp]
    lib.h2o_cache_export.restype = c.c_int
    lib.h2o_cache_export.argtypes = [vp, i32p, c.POINTER(c.c_double), i32p, i32p, c.c_int32, vp]
    lib.h2o_cache_status.restype = c.c_int
    lib.h2o_cache_status.argtypes = [vp, vp]
    lib.h2o_cache_set_decode_shape.restype = c.c_int
    lib.h2o_cache_set_decode_shape.argtypes = [vp, c.c_int32, c.c_int32]
    lib.h2o_cache_set_prefill_path.restype = c.c_int
    lib.h2o_cache_set_decode_path.restype = c.c_int
    lib.h2o_cache_get_decode_path.restype = c.c_int
    lib.h2o_cache_get_decode_path.argtypes = [vp]
    lib.h2o_cache_set_decode_path.argtypes = [vp, c.c_int32]
    lib.h2o_cache_set_prefill_path.argtypes = [vp, c.c_int32]
    lib.h2o_prefill_scratch_layout.restype = c.c_int
    lib.h2o_prefill_scratch_layout.argtypes = [cfgp, c.c_int64, c.POINTER(c.c_size_t)]
    lib.h2o_debug_set_early_prefetch.restype = c.c_int
    lib.h2o_debug_set_early_prefetch.argtypes = [c.c_int32]
    lib.h2o_debug_set_prefill_events.restype = c.c_int
    lib.h2o_debug_set_prefill_events.argtypes = [vp, c.POINTER(vp)]
    lib.h2o_debug_bounds_checked.restype = c.c_int
    lib.h2o_debug_bounds_checked.argtypes = []
    qp = rp = vp  # h2o_queries_t / h2o_ranges_t: by reference, or as packed bytes
    lib.h2o_store_create.restype = c.c_int
    lib.h2o_store_create.argtypes = [c.POINTER(vp), c.POINTER(h2o_store_config_t)]
    lib.h2o_store_destroy.restype = c.c_int
    lib.h2o_store_destroy.argtypes = [vp]
    lib.h2o_debug_store_set_polls.restype = c.c_int
    lib.h2o_debug_store_set_polls.argtypes = [vp, c.c_int32]
    for f in (lib.h2o_store_write, lib.h2o_store_read):
        f.restype = c.c_int
        f.argtypes = [vp, vp, vp, c.c_int32, c.c_int64, c.c_int64, vp, c.c_int64, vp]
    lib.h2o_cross_scratch_bytes.restype = c.c_size_t
    lib.h2o_cross_scratch_bytes.argtypes = [vp, qp, rp]
    lib.h2o_cross_attend.restype = c.c_int
    lib.h2o_cross_attend.argtypes = [vp, qp, rp, vp, c.c_size_t, vp]
    lib.h2o_prefix_scratch_bytes.restype = c.c_size_t
    lib.h2o_prefix_scratch_bytes.argtypes = [vp, qp, rp, c.c_int32, vp, c.c_int32, rp]
    lib.h2o_prefix_attend.restype = c.c_int
    lib.h2o_prefix_attend.argtypes = [vp, qp, rp, c.c_int32, vp, c.c_int32, rp, vp, c.c_size_t, vp]
    lib.h2o_rotate.restype = c.c_int
    lib.h2o_rotate.argtypes = [vp, vp, vp, c.c_int32, c.c_int64, c.c_int32, c.c_int32, c.c_int64, c.c_int64, vp, c.c_int64, c.c_int32, vp]
    lib.h2o_pages_create.restype = c.c_int
    lib.h2o_pages_create.argtypes = [c.POINTER(vp), c.POINTER(h2o_pages_config_t)]
    lib.h2o_pages_destroy.restype = c.c_int
    lib.h2o_pages_destroy.argtypes = [vp]
    lib.h2o_debug_pages_set_polls.restype = c.c_int
    lib.h2o_debug_pages_set_polls.argtypes = [vp, c.c_int32]
    lib.h2o_pages_append.restype = c.c_int
    lib.h2o_pages_append.argtypes = [vp, vp, vp, vp, vp]
    lib.h2o_pages_scratch_bytes.restype = c.c_size_t
    lib.h2o_pages_scratch_bytes.argtypes = [vp, qp, vp, c.c_int32, c.c_int32]
    lib.h2o_pages_attend.restype = c.c_int
    lib.h2o_pages_attend.argtypes = [vp, qp, vp, c.c_int32, c.c_int32, vp, c.c_size_t, vp]
    lib.h2o_strerror.restype = c.c_char_p
    lib.h2o_strerror.argtypes = [c.c_int]
    return lib


lib = _load()


class H2OError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__("%s: %s (%d)" % (where, lib.h2o_strerror(code).decode(), code))


def _check(code: int, where: str):
    if code != H2O_OK:
        raise H2OError(code, where)


def make_config(batch, n_heads, head_dim, dtype, heavy: Sequence[int], recent: Sequence[int], softmax_scale=0.0, device=0,
                query_group=1):
    """Returns (h2o_config_t, keepalive) — the budget arrays must outlive the struct."""
    hv = (ctypes.c_int32 * len(heavy))(*[int(x) for x in heavy])
    rc = (ctypes.c_int32 * len(recent))(*[int(x) for x in recent])
    code = {torch.float32: H2O_F32, torch.bfloat16: H2O_BF16, "f32": H2O_F32, "bf16": H2O_BF16,
            "bf16_kv4": H2O_BF16_KV4}.get(dtype, dtype)
    cfg = h2o_config_t(int(batch), int(n_heads), int(head_dim), int(code), hv, rc, float(softmax_scale), int(device),
                       int(query_group))
    return cfg, (hv, rc)


def h2o_cache_workspace_bytes(cfg: h2o_config_t) -> int:
    return int(lib.h2o_cache_workspace_bytes(ctypes.byref(cfg)))


def h2o_prefill_scratch_bytes(cfg: h2o_config_t, total_tokens: int) -> int:
    return int(lib.h2o_prefill_scratch_bytes(ctypes.byref(cfg), int(total_tokens)))


def _stream_ptr(stream: Optional[torch.cuda.Stream]) -> int:
    if stream is None:
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


class H2OCache:
    """A cache handle plus the torch tensors that back its workspace.

    Methods mirror the C calls one to one: ``prefill_select`` -> h2o_prefill_select,
    ``decode_step`` -> h2o_decode_step, ``export`` -> h2o_cache_export,
    ``status`` -> h2o_cache_status, ``close`` -> h2o_cache_destroy.
    """

    def __init__(self, batch, n_heads, head_dim, dtype, heavy, recent, softmax_scale=0.0, device=0, snapshot=None,
                 query_group=1):
        """``snapshot``: bytes of another handle's workspace (``snapshot()``) to resume from (h2o_cache_attach).
        ``query_group`` > 1: grouped-query attention, q / out carry n_heads * query_group heads."""
        self.cfg, self._keep = make_config(batch, n_heads, head_dim, dtype, heavy, recent, softmax_scale, device,
                                           query_group)
        self.batch, self.n_heads, self.head_dim = int(batch), int(n_heads), int(head_dim)
        self.units = self.batch * self.n_heads
        self.max_B = int(max(int(a) + int(b) for a, b in zip(heavy, recent)))
        self.device = torch.device("cuda", int(device))
        nbytes = h2o_cache_workspace_bytes(self.cfg)
        if nbytes == 0:
            raise H2OError(H2O_ERR_INVALID_ARG, "h2o_cache_workspace_bytes")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        self._ws_ptr = (self.workspace.data_ptr() + 255) // 256 * 256
        self.workspace_bytes = nbytes
        handle = ctypes.c_void_p()
        if snapshot is None:
            _check(lib.h2o_cache_create(ctypes.byref(handle), ctypes.byref(self.cfg), self._ws_ptr, nbytes), "h2o_cache_create")
        else:
            off = self._ws_ptr - self.workspace.data_ptr()
            self.workspace[off:off + nbytes].copy_(snapshot.to(self.device))
            torch.cuda.synchronize(self.device)
            _check(lib.h2o_cache_attach(ctypes.byref(handle), ctypes.byref(self.cfg), self._ws_ptr, nbytes), "h2o_cache_attach")
        self._h = handle
        self._scratch = None

    def snapshot(self):
        """The workspace bytes (a copy): the complete state of the cache.  Synchronises the device first."""
        torch.cuda.synchronize(self.device)
        off = self._ws_ptr - self.workspace.data_ptr()
        return self.workspace[off:off + self.workspace_bytes].clone()

    def prefill_select(self, q, k, v, cu_seqlens, out, stream=None):
        cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        need = h2o_prefill_scratch_bytes(self.cfg, int(cu[-1]))
        if self._scratch is None or self._scratch.numel() < need + 256:
            self._scratch = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        sp = (self._scratch.data_ptr() + 255) // 256 * 256
        _check(lib.h2o_prefill_select(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                      cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), out.data_ptr(), sp, need,
                                      _stream_ptr(stream)), "h2o_prefill_select")

    def prefill_select_static(self, q, k, v, cu_seqlens, out, stream=None):
        """h2o_prefill_select_static: the scratch is the library's built-in array, nothing is allocated here."""
        cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        _check(lib.h2o_prefill_select_static(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                             cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), out.data_ptr(),
                                             _stream_ptr(stream)), "h2o_prefill_select_static")

    def decode_step(self, q, k_new, v_new, out, evicted_pos=None, stream=None):
        _check(lib.h2o_decode_step(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(),
                                   None if evicted_pos is None else evicted_pos.data_ptr(), _stream_ptr(stream)),
               "h2o_decode_step")

    def decode_chunk(self, q, k, v, out, evicted_pos=None, stream=None):
        """h2o_decode_chunk: q, k, v, out are [n_tokens, batch, n_heads, head_dim]; evicted_pos [n_tokens, batch, n_heads]."""
        _check(lib.h2o_decode_chunk(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(), int(q.shape[0]), out.data_ptr(),
                                    None if evicted_pos is None else evicted_pos.data_ptr(), _stream_ptr(stream)),
               "h2o_decode_chunk")

    def set_chunk_path(self, path: int):
        _check(lib.h2o_cache_set_chunk_path(self._h, int(path)), "h2o_cache_set_chunk_path")

    def set_score_mode(self, mode: int):
        """0: rank by the accumulated score, 1: by the averaged score (empty cache only)."""
        _check(lib.h2o_cache_set_score_mode(self._h, int(mode)), "h2o_cache_set_score_mode")

    def set_mask(self, kind: int, a: int = 1, b: int = 0):
        """h2o_cache_set_mask: 0 none, 1 strided(stride a, local window b), 2 fixed(block a, b summary columns)."""
        _check(lib.h2o_cache_set_mask(self._h, int(kind), int(a), int(b)), "h2o_cache_set_mask")

    def set_topk(self, m: int):
        """h2o_cache_set_topk: in decode steps a query attends only its m largest logits (0 = off)."""
        _check(lib.h2o_cache_set_topk(self._h, int(m)), "h2o_cache_set_topk")

    def fscore(self, hkind: int = 0, stream=None):
        """F_score per (sequence, head): sum of h(accumulated score); h: 0 identity, 1 sqrt(z+1), 2 log(z+1)."""
        out = torch.empty(self.cfg.batch * self.cfg.n_heads, dtype=torch.float64, device=self.device)
        _check(lib.h2o_cache_fscore(self._h, int(hkind), out.data_ptr(), _stream_ptr(stream)), "h2o_cache_fscore")
        return out.view(self.cfg.batch, self.cfg.n_heads)

    def reset(self, stream=None):
        _check(lib.h2o_cache_reset(self._h, _stream_ptr(stream)), "h2o_cache_reset")

    def _staging(self, tokens: int):
        need = int(lib.h2o_host_staging_bytes(ctypes.byref(self.cfg), int(tokens)))
        st = getattr(self, "_stage", None)
        if st is None or st.numel() < need + 256:
            self._stage = st = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        return (st.data_ptr() + 255) // 256 * 256, need

    def prefill_select_host(self, q, k, v, cu_seqlens, out, stream=None):
        """Host (ideally pinned) tensors in and out; the copies run on the stream inside the C call."""
        cu = np.ascontiguousarray(cu_seqlens, dtype=np.int32)
        need = h2o_prefill_scratch_bytes(self.cfg, int(cu[-1]))
        if self._scratch is None or self._scratch.numel() < need + 256:
            self._scratch = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
        sp = (self._scratch.data_ptr() + 255) // 256 * 256
        sg, sg_bytes = self._staging(int(cu[-1]))
        _check(lib.h2o_prefill_select_host(self._h, q.data_ptr(), k.data_ptr(), v.data_ptr(),
                                           cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), out.data_ptr(), sg, sg_bytes,
                                           sp, need, _stream_ptr(stream)), "h2o_prefill_select_host")

    def decode_step_host(self, q, k_new, v_new, out, evicted_pos=None, stream=None):
        if getattr(self, "_dstage", None) is None:
            need = int(lib.h2o_host_staging_bytes(ctypes.byref(self.cfg), self.batch))
            buf = torch.empty(need + 256, dtype=torch.uint8, device=self.device)
            self._dstage = (buf, (buf.data_ptr() + 255) // 256 * 256, need)
        _, sg, sg_bytes = self._dstage
        _check(lib.h2o_decode_step_host(self._h, q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), out.data_ptr(),
                                        None if evicted_pos is None else evicted_pos.data_ptr(), sg, sg_bytes,
                                        _stream_ptr(stream)), "h2o_decode_step_host")

    def export(self, stream=None):
        """(pos [units, max_B] int32 with -1 padding, acc [units, max_B] float64, count [units], t [units])."""
        pitch = self.max_B
        pos = np.empty((self.units, pitch), dtype=np.int32)
        acc = np.empty((self.units, pitch), dtype=np.float64)
        count = np.empty(self.units, dtype=np.int32)
        t = np.empty(self.units, dtype=np.int32)
        i32p = ctypes.POINTER(ctypes.c_int32)
        _check(lib.h2o_cache_export(self._h, pos.ctypes.data_as(i32p), acc.ctypes.data_as(ctypes.POINTER(ctypes.c_double)),
                                    count.ctypes.data_as(i32p), t.ctypes.data_as(i32p), pitch, _stream_ptr(stream)),
               "h2o_cache_export")
        return pos, acc, count, t

    def set_decode_shape(self, split: int = 0, stages: int = 0):
        _check(lib.h2o_cache_set_decode_shape(self._h, int(split), int(stages)), "h2o_cache_set_decode_shape")

    def set_prefill_events(self, events):
        """h2o_debug_set_prefill_events: four torch.cuda.Event(enable_timing=True), already recorded once (torch
        creates the CUDA handle lazily), for the next prefill_select call."""
        arr = (ctypes.c_void_p * 4)(*[int(e.cuda_event) for e in events])
        _check(lib.h2o_debug_set_prefill_events(self._h, arr), "h2o_debug_set_prefill_events")

    def set_decode_path(self, path: int):
        _check(lib.h2o_cache_set_decode_path(self._h, int(path)), "h2o_cache_set_decode_path")

    def decode_path(self) -> int:
        return int(lib.h2o_cache_get_decode_path(self._h))

    def set_prefill_path(self, path: int):
        _check(lib.h2o_cache_set_prefill_path(self._h, int(path)), "h2o_cache_set_prefill_path")

    def prefill_column_sums(self, total_tokens: int):
        """acc0 of the last prefill_select as a [n_heads, total_tokens] float64 tensor (a view of the scratch)."""
        acc_off = ctypes.c_size_t()
        _check(lib.h2o_prefill_scratch_layout(ctypes.byref(self.cfg), int(total_tokens), ctypes.byref(acc_off)),
               "h2o_prefill_scratch_layout")
        base = (self._scratch.data_ptr() + 255) // 256 * 256 - self._scratch.data_ptr()
        n = self.n_heads * int(total_tokens)
        raw = self._scratch[base + acc_off.value: base + acc_off.value + 8 * n]
        return raw.view(torch.float64).view(self.n_heads, int(total_tokens))

    def status(self, stream=None) -> int:
        return int(lib.h2o_cache_status(self._h, _stream_ptr(stream)))

    def close(self):
        if getattr(self, "_h", None) is not None:
            lib.h2o_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


_DTYPES = {torch.float32: H2O_F32, torch.bfloat16: H2O_BF16}
# h2o_queries_t and h2o_ranges_t as bytes: a step's host time counts, and packing costs a third of filling a Structure
_pack_queries = struct.Struct("@PPPPqqqfiiii0P").pack
_pack_ranges = struct.Struct("@PPi0P").pack
_raw_stream = torch._C._cuda_getCurrentRawStream


def _bad(why: str):
    raise ValueError("H2OStore: " + why)


def _rows_alike(k, v, rows, heads, dim):
    """Strides of k and v [rows, heads, dim]: dense heads and one row stride, as far as there is more than one of them.  A
    broadcast over the rows is refused (a stride of 0 means dense to the library)."""
    if rows == 0 or (k == v and k[2] == 1 and k[1] == dim and k[0] > 0):
        return True
    return k[2] == v[2] == 1 and (heads == 1 or k[1] == v[1] == dim) and (rows == 1 or k[0] == v[0] > 0)


class H2OStore:
    """K/V rows that many queries read and nothing evicts (h2o_store_*): an encoder's states, a prompt that a batch
    shares, a sequence's own tokens.

    ``k``, ``v``: float32 or bfloat16 [rows, heads, head_dim] (rows may be strided), or uint8 e4m3 codes
    [heads, rows, head_dim] with ``k_scale``, ``v_scale`` uint8 [heads, rows] (value = code * 2^(scale - 127), scales
    outside 112 .. 134 as the nearer of the two).  The tensors stay the caller's (this
    object keeps a reference) and are read where they lie.  Methods mirror the C calls: ``write`` ->
    h2o_store_write, ``read`` -> h2o_store_read, ``cross_attend`` -> h2o_cross_attend, ``prefix_attend`` ->
    h2o_prefix_attend, ``close`` -> h2o_store_destroy.  Results go to tensors that the caller passes; scratch comes
    from torch's allocator on the call's stream, one piece per call.
    """

    def __init__(self, k, v, k_scale=None, v_scale=None):
        if not k.is_cuda or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device or k.dim() != 3:
            _bad("k and v must be CUDA tensors of one 3-d shape, dtype and device")
        eight = k.dtype == torch.uint8
        if eight:
            self.n_heads, self.rows, self.head_dim = k.shape
            if not k.is_contiguous() or not v.is_contiguous():
                _bad("8-bit k and v must be contiguous")
            for s in (k_scale, v_scale):
                if s is None or s.dtype != torch.uint8 or s.shape != k.shape[:2] or not s.is_contiguous() or s.device != k.device:
                    _bad("8-bit rows need contiguous uint8 scales [heads, rows] on the same device")
        else:
            if k.dtype not in _DTYPES:
                _bad("k and v must be float32, bfloat16 or uint8")
            if k_scale is not None or v_scale is not None:
                _bad("scales belong to 8-bit rows")
            self.rows, self.n_heads, self.head_dim = k.shape
            if not _rows_alike(k.stride(), v.stride(), *k.shape):
                _bad("rows of k and v must have one stride and dense heads")
        self.format = H2O_KV8 if eight else _DTYPES[k.dtype]
        self.device = k.device
        self._index = k.device.index
        self._need = {}  # scratch bytes by the sizes of a call
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()  # the zero is there, whatever stream comes next
        cfg = h2o_store_config_t(self.n_heads, self.head_dim, self.format, self.device.index, self.rows,
                                 0 if eight or self.rows <= 1 else k.stride(0), k.data_ptr(), v.data_ptr(),
                                 k_scale.data_ptr() if eight else None, v_scale.data_ptr() if eight else None,
                                 self._status.data_ptr())
        self._h = None
        handle = ctypes.c_void_p()
        _check(lib.h2o_store_create(ctypes.byref(handle), ctypes.byref(cfg)), "h2o_store_create")
        self._h = handle

    @classmethod
    def empty_kv8(cls, rows: int, n_heads: int, head_dim: int, device=0):
        """A store of 8-bit rows, all zero."""
        dev = torch.device("cuda", device) if isinstance(device, int) else device
        k = torch.zeros((n_heads, rows, head_dim), dtype=torch.uint8, device=dev)
        scale = torch.full((n_heads, rows), 127, dtype=torch.uint8, device=dev)
        return cls(k, torch.zeros_like(k), scale, scale.clone())

    # ---- argument checks ----
    def _rows(self, k, v, rows, first_row):
        shape = k.shape
        if len(shape) != 3 or v.shape != shape or shape[1] != self.n_heads or shape[2] != self.head_dim:
            _bad("k and v must be [tokens, %d, %d]" % (self.n_heads, self.head_dim))
        dtype = _DTYPES.get(k.dtype)
        if dtype is None or v.dtype is not k.dtype or k.get_device() != self._index or v.get_device() != self._index:
            _bad("k and v must both be float32 or bfloat16 on %s" % self.device)
        n, stride = shape[0], k.stride()
        if not _rows_alike(stride, v.stride(), *shape):
            _bad("k and v must have one token stride and dense heads")
        if rows is not None and (rows.dtype is not torch.int64 or rows.shape != (n,) or rows.get_device() != self._index or not rows.is_contiguous()):
            _bad("rows must be a contiguous int64 [tokens] on %s" % self.device)
        return (self._h, k.data_ptr(), v.data_ptr(), dtype, n, stride[0] if n > 1 else 0,
                None if rows is None else rows.data_ptr(), first_row)

    def _queries(self, q, out, cu_q, max_q, lse, softmax_scale, batch):
        shape = q.shape
        if len(shape) != 3 or shape[2] != self.head_dim or shape[1] < self.n_heads or shape[1] % self.n_heads:
            _bad("q must be [tokens, multiple of %d, %d]" % (self.n_heads, self.head_dim))
        tokens, heads, dim = shape
        dtype = _DTYPES.get(q.dtype)
        if dtype is None or out.dtype is not q.dtype or out.shape != shape:
            _bad("q and out must be float32 or bfloat16 of one shape and dtype")
        if q.get_device() != self._index or out.get_device() != self._index:
            _bad("q and out must be on %s" % self.device)
        s, o = q.stride(), out.stride()
        if tokens and (s[2] != 1 or o[2] != 1 or (heads > 1 and (s[1] != dim or o[1] != dim))):
            _bad("q and out must have dense heads")
        if tokens > 1 and (s[0] == 0 or o[0] == 0):  # (0 means dense to the library)
            _bad("q and out must not be broadcast over the tokens")
        if cu_q is None:
            if max_q != 1 or tokens < batch:
                _bad("without cu_q there is one token per sequence")
        elif cu_q.dtype is not torch.int32 or cu_q.shape != (batch + 1,) or cu_q.get_device() != self._index or not cu_q.is_contiguous():
            _bad("cu_q must be a contiguous int32 [batch + 1] on %s" % self.device)
        if lse is not None and (lse.dtype is not torch.float32 or lse.shape != (tokens, heads) or lse.get_device() != self._index or not lse.is_contiguous()):
            _bad("lse must be a contiguous float32 [tokens, heads] on %s" % self.device)
        group = heads // self.n_heads
        return (_pack_queries(q.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr(), 0 if cu_q is None else cu_q.data_ptr(),
                              tokens, s[0] if tokens > 1 else 0, o[0] if tokens > 1 else 0, softmax_scale, dtype, group, batch, max_q),
                (tokens, group, dtype, batch, max_q))

    def _ranges(self, begin, length, most, count):
        if begin.dtype is not torch.int64 or length.dtype is not torch.int32 or begin.shape != (count,) or length.shape != (count,):
            _bad("begin must be int64 and length int32, one entry per range")
        if begin.get_device() != self._index or length.get_device() != self._index or not begin.is_contiguous() or not length.is_contiguous():
            _bad("begin and length must be contiguous on %s" % self.device)
        return _pack_ranges(begin.data_ptr(), length.data_ptr(), most)

    def _scratch(self, nbytes, stream):
        """A piece of scratch of this call's own, on its stream; torch's blocks are 512-byte aligned."""
        if stream is None:
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        with torch.cuda.stream(stream):
            return torch.empty(nbytes, dtype=torch.uint8, device=self.device)

    def _needs(self, sizes, nbytes):
        """Remembers how much scratch a call of these sizes needs (a function of the sizes alone, which a call that went
        through has shown to be valid)."""
        if sizes not in self._need:
            if len(self._need) >= 1024:
                self._need.clear()
            self._need[sizes] = nbytes

    # ---- calls ----
    def write(self, k, v, rows=None, first_row=0, stream=None):
        """Quantise k, v [tokens, heads, head_dim] into store rows ``rows`` (int64, device) or first_row, first_row + 1, ..."""
        code = lib.h2o_store_write(*self._rows(k, v, rows, first_row), _raw_stream(self._index) if stream is None else stream.cuda_stream)
        if code:
            _check(code, "h2o_store_write")

    def read(self, k, v, rows=None, first_row=0, stream=None):
        """Read store rows back into k, v [tokens, heads, head_dim]."""
        code = lib.h2o_store_read(*self._rows(k, v, rows, first_row), _raw_stream(self._index) if stream is None else stream.cuda_stream)
        if code:
            _check(code, "h2o_store_read")

    def cross_attend(self, q, begin, length, out, max_len, cu_q=None, max_q=1, lse=None, softmax_scale=0.0, stream=None):
        """Sequence b's query tokens attend store rows begin[b] .. begin[b] + length[b] - 1.  q, out: [tokens, query
        heads, head_dim]; cu_q: int32 [batch + 1] first token of each sequence (None: token b is sequence b); max_q,
        max_len: upper bounds; lse: float32 [tokens, query heads] or None."""
        batch = begin.shape[0] if begin.dim() == 1 else -1
        qs, sizes = self._queries(q, out, cu_q, max_q, lse, softmax_scale, batch)
        rs = self._ranges(begin, length, max_len, batch)
        sizes += (max_len,)
        need = self._need.get(sizes)
        if need is None:
            need = lib.h2o_cross_scratch_bytes(self._h, qs, rs)
        scratch = self._scratch(need, stream) if need else None
        code = lib.h2o_cross_attend(self._h, qs, rs, scratch.data_ptr() if need else None, need,
                                    _raw_stream(self._index) if stream is None else stream.cuda_stream)
        if code:
            _check(code, "h2o_cross_attend")
        self._needs(sizes, need)

    def prefix_attend(self, q, prefix_begin, prefix_len, own_begin, own_len, out, max_prefix, max_own, cu_group=None,
                      max_group=0, cu_q=None, max_q=1, lse=None, softmax_scale=0.0, stream=None):
        """Groups of consecutive sequences (cu_group: int32 [groups + 1], None: one group) share the store rows
        prefix_begin[g] .. + prefix_len[g] - 1; sequence b's own rows are own_begin[b] .. + own_len[b] - 1, the last
        of them those of its query tokens.  max_group: upper bound of a group's sequences (0: the batch)."""
        batch = own_begin.shape[0] if own_begin.dim() == 1 else -1
        groups = prefix_begin.shape[0] if prefix_begin.dim() == 1 else -1
        if cu_group is None:
            if groups != 1:
                _bad("several groups need cu_group")
            cg = None
        else:
            if cu_group.dtype is not torch.int32 or cu_group.shape != (groups + 1,) or cu_group.get_device() != self._index or not cu_group.is_contiguous():
                _bad("cu_group must be a contiguous int32 [groups + 1] on %s" % self.device)
            cg = cu_group.data_ptr()
        qs, sizes = self._queries(q, out, cu_q, max_q, lse, softmax_scale, batch)
        ps = self._ranges(prefix_begin, prefix_len, max_prefix, groups)
        os_ = self._ranges(own_begin, own_len, max_own, batch)
        most = max_group or max(1, batch)
        sizes += (max_prefix, max_own, groups, most)
        need = self._need.get(sizes)
        if need is None:
            need = lib.h2o_prefix_scratch_bytes(self._h, qs, ps, groups, cg, most, os_)
        scratch = self._scratch(need, stream) if need else None
        code = lib.h2o_prefix_attend(self._h, qs, ps, groups, cg, most, os_, scratch.data_ptr() if need else None, need,
                                     _raw_stream(self._index) if stream is None else stream.cuda_stream)
        if code:
            _check(code, "h2o_prefix_attend")
        self._needs(sizes, need)

    def status(self) -> int:
        """H2O_OK, or the H2O_ERR_* a kernel recorded (synchronises)."""
        return int(self._status.item())

    def close(self):
        if getattr(self, "_h", None) is not None:
            lib.h2o_store_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class _NoPages:
    """Stands where the _pages extension should be: whatever is asked of it says why it is not there."""

    def __init__(self, why):
        self._why = why

    def __getattr__(self, name):
        raise ImportError(self._why)


def _load_pages():
    at = pages_path()
    if not os.path.exists(at):
        return _NoPages(os.path.basename(at) + " is not built, which H2ORotary and H2OPages need with this Python and torch (run "
                        "`python paper_2306_14048_b200/build.py`); there is no fallback path")
    spec = importlib.util.spec_from_file_location(__package__ + "._pages", at)
    try:
        _pages = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(_pages)
    except ImportError as e:
        return _NoPages("%s does not load (%s): build it again (`python paper_2306_14048_b200/build.py --force`); there is no fallback path"
                        % (os.path.basename(at), e))
    _pages.bind(*[ctypes.cast(f, ctypes.c_void_p).value
                  for f in (lib.h2o_rotate, lib.h2o_pages_append, lib.h2o_pages_scratch_bytes, lib.h2o_pages_attend)])
    return _pages


# checks of arguments of the calls below, packing and the call itself, in C++ (csrc/pages_binding.cpp): a step's host time counts
_pages = _load_pages()


def _wrong(who: str, why: str):
    raise ValueError(who + ": " + why)


def _raw_of(stream, index, who):
    """The handle of a stream that a caller passes, which has to be of the object's device."""
    if getattr(stream, "device_index", index) != index:
        _wrong(who, "stream must be of device %d" % index)
    return stream.cuda_stream


_NO_TURN = (0, 0, 0, 0)


class _Lasting:
    """Small tensors on the device that belong to an object and that its calls' kernels use: when the object goes, torch's allocator
    gives their memory to others only after what has been enqueued on every stream that a call has used (once per stream, noted by the
    first call).  Streams that torch does not own may be gone by then: a call on one needs the object until it has run."""

    def _keep(self, *tensors):
        self._kept, self._streams = tensors, {_raw_stream(self._index)}

    def _note(self, raw, stream):
        self._streams.add(raw)
        if stream is None:
            stream = torch.cuda.current_stream(self.device)
        if isinstance(stream, torch.cuda.Stream) and (raw == 0 or stream.stream_id != raw):  # (another library's has its address as its id)
            for t in self._kept:
                t.record_stream(stream)


class H2ORotary(_Lasting):
    """Rotary positions of heads (h2o_rotate): pairs of channels turned by position * frequency.

    ``frequencies``: radians per position of each of the rotary_dim / 2 pairs (None: base ** (-2 i / rotary_dim));
    ``axes``: which axis of the positions each pair follows (None: one axis); ``pairs``: "halves" (channels i and
    i + rotary_dim / 2) or "neighbours" (channels 2 i and 2 i + 1).  rotary_dim: the first channels of a head, all of them
    by default; the others stay as they are.  The two small tables are kept on the device by this object:
    making it copies them there and waits for the copy, so a program makes one for each kind of layer and keeps it.  It may go once
    its last call has been made (on a stream that torch does not own: has run); a captured graph needs it for as long as it is replayed.
    """

    def __init__(self, head_dim: int, rotary_dim: Optional[int] = None, base: float = 10000.0, frequencies=None, axes=None,
                 pairs: str = "halves", device=0):
        _pages.rotate  # (says so where the extension is missing)
        self.head_dim = int(head_dim)
        self.rotary_dim = self.head_dim if rotary_dim is None else int(rotary_dim)
        if self.head_dim < 8 or self.head_dim > 512 or self.head_dim % 8:
            _wrong("H2ORotary", "head_dim must be a multiple of 8, up to 512")
        if not 2 <= self.rotary_dim <= self.head_dim or self.rotary_dim % 2:
            _wrong("H2ORotary", "rotary_dim must be even, 2 .. head_dim")
        half = self.rotary_dim // 2
        if frequencies is None:
            frequencies = [float(base) ** (-2.0 * i / self.rotary_dim) for i in range(half)]
        frequencies = np.ascontiguousarray(np.asarray(frequencies, dtype=np.float64))
        if frequencies.shape != (half,) or not np.isfinite(frequencies).all():
            _wrong("H2ORotary", "frequencies must be %d finite numbers" % half)
        self.axes = 1
        if axes is not None:
            axes = np.asarray(axes)
            if axes.shape != (half,) or axes.dtype.kind not in "iu" or axes.min() < 0 or axes.max() > 7:
                _wrong("H2ORotary", "axes must be %d whole numbers, 0 .. 7" % half)
            self.axes = int(axes.max()) + 1
        if pairs not in ("halves", "neighbours"):
            _wrong("H2ORotary", "pairs must be 'halves' or 'neighbours'")
        self.device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        if self.device.type != "cuda":
            _wrong("H2ORotary", "a CUDA device is needed; there is no fallback")
        self._frequency = torch.from_numpy(frequencies).to(self.device)
        self.device, self._index = self._frequency.device, self._frequency.device.index
        self._axis = None if self.axes == 1 else torch.from_numpy(axes.astype(np.uint8)).to(self.device)
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()  # the tables are there, whatever stream comes next
        self._c = h2o_rotary_t(self._frequency.data_ptr(), None if self._axis is None else self._axis.data_ptr(), self.rotary_dim, self.axes,
                               0 if pairs == "halves" else 1, self._index, self._status.data_ptr())
        self._at = ctypes.addressof(self._c)
        self._turn = (self._at, self._index, self.head_dim, self.axes)  # what an append passes on
        self._keep(*[t for t in (self._frequency, self._axis, self._status) if t is not None])

    def apply(self, x, positions, out, inverse=False, stream=None):
        """Rotates x [tokens, heads, head_dim] into out (which may be x).  inverse: takes the rotation back, which is also
        the gradient of a rotation with respect to its input."""
        raw = _raw_stream(self._index) if stream is None else _raw_of(stream, self._index, "H2ORotary")
        if raw not in self._streams:
            self._note(raw, stream)
        code = _pages.rotate(self._at, self._index, self.head_dim, self.axes, x, positions, out, inverse, raw)
        if code:
            _check(code, "h2o_rotate")

    status = H2OStore.status


def _pool_strides(k, v):
    """Elements between pages, rows, heads and channels of a pool's k and v [pages, page_size, heads, head_dim]."""
    shape, strides = k.shape, list(k.stride())
    used = [i for i in range(4) if shape[i] > 1]
    if any(strides[i] != v.stride(i) for i in used) or (3 in used and strides[3] != 1):
        _wrong("H2OPages", "k and v must have the same strides and dense channels")
    if any(strides[i] == 0 for i in used):  # (three zeros mean dense to the library)
        _wrong("H2OPages", "k and v must not be broadcast over the pages, rows or heads")
    if shape[2] == 1:  # strides that are never used
        strides[2] = shape[3]
    if shape[0] == 1:
        strides[0] = max(strides[1] * shape[1], strides[2] * shape[2])
    return strides


class H2OPages(_Lasting):
    """A paged K/V cache (h2o_pages_*): rows in pages of a pool, a table of pages for each sequence.

    ``k``, ``v``: float32 or bfloat16 [pages, page_size, heads, head_dim] of the same strides, channels dense (any order of the
    other three: a pool [pages, heads, page_size, head_dim] is given as its transpose(1, 2), one of K and V together as its
    parts).  page_size: a multiple of 8.  The tensors stay the caller's (this object keeps a reference).  ``table``: int32 [batch,
    most pages of a sequence], an entry outside the pool is no page; ``length``: int32 [batch], rows of each sequence, those
    of the call's tokens included, which are its last ones.  Methods mirror the C calls: ``append`` ->
    h2o_pages_append, ``attend`` -> h2o_pages_attend, ``close`` -> h2o_pages_destroy.  Results go to tensors that the caller
    passes; scratch comes from torch's allocator on the call's stream, one piece per call.
    A captured graph needs the object, and the rotary it was captured with, for as long as it is replayed.
    """

    def __init__(self, k, v):
        _pages.attend  # (says so where the extension is missing)
        if not k.is_cuda or k.dim() != 4 or k.shape != v.shape or k.dtype != v.dtype or k.device != v.device:
            _wrong("H2OPages", "k and v must be CUDA tensors of one 4-d shape, dtype and device")
        if k.dtype not in _DTYPES:
            _wrong("H2OPages", "k and v must be float32 or bfloat16")
        self.n_pages, self.page_size, self.n_heads, self.head_dim = k.shape
        strides = _pool_strides(k, v)
        self.format = _DTYPES[k.dtype]
        self.device, self._index = k.device, k.device.index
        self.k, self.v = k, v
        self._status = torch.zeros(1, dtype=torch.int32, device=self.device)
        torch.cuda.current_stream(self.device).synchronize()  # the zero is there, whatever stream comes next
        cfg = h2o_pages_config_t(self.n_heads, self.head_dim, self.format, self._index, self.n_pages, self.page_size, strides[0], strides[1],
                                 strides[2], k.data_ptr(), v.data_ptr(), self._status.data_ptr())
        self._h = None
        handle = ctypes.c_void_p()
        _check(lib.h2o_pages_create(ctypes.byref(handle), ctypes.byref(cfg)), "h2o_pages_create")
        self._h = handle
        self._at = handle.value
        self._keep(self._status)

    def append(self, k, v, table, length, cu=None, rotary=None, positions=None, q=None, q_out=None, stream=None):
        """Appends k, v [tokens, heads, head_dim] to their sequences' pages; with ``rotary`` k is rotated on the way, and q
        [tokens, query heads, head_dim] into q_out (which may be q).  cu: int32 [batch + 1] first token of each sequence (None:
        token b is sequence b); positions: as for H2ORotary.apply (None: each token's row, on every axis)."""
        raw = _raw_stream(self._index) if stream is None else _raw_of(stream, self._index, "H2OPages")
        if raw not in self._streams:
            self._note(raw, stream)
        turn = _NO_TURN
        if rotary is not None:
            turn = rotary._turn
            if raw not in rotary._streams:
                rotary._note(raw, stream)
        code = _pages.append(self._at, self._index, self.n_heads, self.head_dim, self.format, k, v, table, length, cu, *turn, positions, q, q_out, raw)
        if code:
            _check(code, "h2o_pages_append")

    def attend(self, q, table, length, out, max_len, window=0, sinks=0, cu=None, max_q=1, lse=None, softmax_scale=0.0, stream=None):
        """Each sequence's query tokens attend its rows up to their own, with ``window`` > 0 the last ``window`` of them (their own
        included) and the sequence's first ``sinks``.  q, out: [tokens, query heads, head_dim]; cu: int32 [batch + 1] first
        token of each sequence (None: token b is sequence b); max_q, max_len: upper bounds of a sequence's tokens and rows;
        lse: float32 [tokens, query heads] or None."""
        if stream is not None:  # its scratch, too, comes from that stream
            _raw_of(stream, self._index, "H2OPages")
            with torch.cuda.stream(stream):
                return self.attend(q, table, length, out, max_len, window, sinks, cu, max_q, lse, softmax_scale)
        raw = _raw_stream(self._index)
        if raw not in self._streams:
            self._note(raw, None)
        code = _pages.attend(self._at, self._index, self.n_heads, self.head_dim, self.format, q, table, length, out, max_len, window, sinks, cu, max_q,
                             lse, softmax_scale, raw)
        if code:
            _check(code, "h2o_pages_attend")

    status = H2OStore.status

    def close(self):
        if getattr(self, "_h", None) is not None:
            lib.h2o_pages_destroy(self._h)
            self._h, self._at = None, 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
