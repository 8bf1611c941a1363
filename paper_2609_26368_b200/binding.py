"""Thin ctypes binding of ``libhs2.so``: argument marshalling only.

Every step of the path runs inside the CUDA library; this module turns torch tensors into
device pointers, fills the ``hs2_problem`` struct, allocates outputs / scratch with torch when the
caller did not pass them, and raises on a non-zero status.  There is no fallback: a missing
library or a missing GPU is an error.
"""
from __future__ import annotations

import ctypes as C
import os
import functools
import struct
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libhs2.so")

HS2_OK, HS2_ERR_INVALID_ARG, HS2_ERR_UNSUPPORTED, HS2_ERR_WORKSPACE_TOO_SMALL, HS2_ERR_CUDA, \
    HS2_ERR_STATIC_SCRATCH = range(6)
HS2_STATIC_DECODE_MAX_PAIRS = 64
HS2_F32, HS2_BF16 = 0, 1
HS2_OP_FULL_ATTN_SELECT, HS2_OP_TOPK_SELECT, HS2_OP_SPARSE_ATTN_PREFILL, HS2_OP_SPARSE_ATTN_DECODE = range(4)
HS2_OP_FULL_ATTN_SELECT_FP8KV, HS2_OP_WINDOW_ATTN = 4, 5
HS2_MAX_PAGE_REGIONS = 8

EXPORTS = ["hs2_workspace_bytes", "hs2_full_attn_select", "hs2_topk_select", "hs2_sparse_attn_prefill",
           "hs2_sparse_attn_decode", "hs2_sparse_attn_prefill_gated", "hs2_sparse_attn_decode_gated",
           "hs2_sparse_attn_prefill_fp8kv", "hs2_sparse_attn_decode_fp8kv", "hs2_full_attn_select_fp8kv", "hs2_kv_project",
           "hs2_kv_project_fp8_records",
           "hs2_sparse_attn_decode_static", "hs2_probe_gather", "hs2_status_string", "hs2_last_cuda_error",
           "hs2_launch_count", "hs2_device_error_flags", "hs2_set_filter_min_keys", "hs2_set_tcgen05_enabled",
           "hs2_window_attn", "hs2_paged_workspace_bytes", "hs2_paged_attn_decode", "hs2_paged_attn_decode_fp8kv",
           "hs2_pages_workspace_bytes", "hs2_pages_reserve", "hs2_pages_write", "hs2_pages_fork", "hs2_pages_free",
           "hs2_pages_compact", "hs2_pages_copy"]


class HS2Error(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        super().__init__("%s: %s%s" % (where, hs2_status_string(status), detail))


class _CProblem(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("q_len", C.c_int32), ("kv_len", C.c_int32),
                ("k_sel", C.c_int32), ("window", C.c_int32), ("softmax_scale", C.c_float),
                ("dtype", C.c_int), ("q_start", C.c_void_p), ("kv_lens", C.c_void_p),
                ("q_stride", C.c_int64 * 3), ("kv_stride", C.c_int64 * 3), ("o_stride", C.c_int64 * 3),
                ("select_block", C.c_int32), ("kv_scale_stride", C.c_int64 * 3)]


class _CPagedProblem(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("max_pages", C.c_int32), ("window", C.c_int32),
                ("n_first", C.c_int32), ("softmax_scale", C.c_float), ("dtype", C.c_int), ("page_table", C.c_void_p),
                ("table_stride", C.c_int64), ("kv_lens", C.c_void_p), ("q_stride", C.c_int64 * 2), ("o_stride", C.c_int64 * 2),
                ("kv_stride", C.c_int64 * 3), ("kv_scale_stride", C.c_int64 * 3)]


class _CPagePool(C.Structure):
    _fields_ = [("n_pages", C.c_int32), ("page_size", C.c_int32), ("max_seqs", C.c_int32), ("max_pages", C.c_int32),
                ("ref_counts", C.c_void_p), ("page_table", C.c_void_p), ("lens", C.c_void_p)]


class _CPageRegion(C.Structure):
    _fields_ = [("base", C.c_void_p), ("n_layers", C.c_int32), ("row_bytes", C.c_int32), ("layer_stride", C.c_int64),
                ("page_stride", C.c_int64), ("token_stride", C.c_int64)]


_lib = None


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """dlopen the in-tree library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError("%s is missing: build it with `python -m paper_2609_26368_b200.build`" % _LIB_PATH)
        lib = C.CDLL(_LIB_PATH)
        lib.hs2_workspace_bytes.restype = C.c_size_t
        lib.hs2_workspace_bytes.argtypes = [C.POINTER(_CProblem), C.c_int]
        lib.hs2_status_string.restype = C.c_char_p
        lib.hs2_status_string.argtypes = [C.c_int]
        lib.hs2_last_cuda_error.restype = C.c_int
        lib.hs2_launch_count.restype = C.c_ulonglong
        vp, sz = C.c_void_p, C.c_size_t
        pp = C.POINTER(_CProblem)
        lib.hs2_full_attn_select.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_topk_select.argtypes = [pp, vp, vp, vp, sz, vp]
        lib.hs2_sparse_attn_prefill.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_sparse_attn_decode.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_sparse_attn_decode_static.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.hs2_sparse_attn_prefill_gated.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_sparse_attn_decode_gated.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_kv_project.argtypes = [C.c_int64, C.c_int32, C.c_int32, vp, C.c_int64, vp, C.c_int64, vp, C.c_int64, vp, vp]
        lib.hs2_kv_project.restype = C.c_int
        lib.hs2_kv_project_fp8_records.argtypes = [C.c_int64, C.c_int32, C.c_int32, vp, C.c_int64, vp, C.c_int64, vp, C.c_int64,
                                                   C.c_int64, vp, C.c_int64, C.c_int64, vp]
        lib.hs2_kv_project_fp8_records.restype = C.c_int
        lib.hs2_sparse_attn_prefill_fp8kv.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.hs2_sparse_attn_decode_fp8kv.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        lib.hs2_full_attn_select_fp8kv.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_probe_gather.argtypes = [pp, vp, vp, vp, C.c_int, vp, vp]
        lib.hs2_probe_gather.restype = C.c_int
        lib.hs2_window_attn.argtypes = [vp, C.c_int32, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        gp = lp = rp = vp   # packed bytes, or byref of the structs above
        i32 = C.c_int32
        lib.hs2_paged_workspace_bytes.restype = sz
        lib.hs2_paged_workspace_bytes.argtypes = [gp]
        lib.hs2_paged_attn_decode.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_paged_attn_decode_fp8kv.argtypes = [gp, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.hs2_pages_workspace_bytes.restype = sz
        lib.hs2_pages_workspace_bytes.argtypes = [lp, i32]
        lib.hs2_pages_reserve.argtypes = [lp, rp, i32, vp, vp, i32, vp, vp, sz, vp]
        lib.hs2_pages_write.argtypes = [lp, rp, i32, vp, vp, vp, vp, vp, i32, i32, vp]
        lib.hs2_pages_fork.argtypes = [lp, vp, vp, i32, vp, sz, vp]
        lib.hs2_pages_free.argtypes = [lp, vp, vp, i32, vp]
        lib.hs2_pages_compact.argtypes = [lp, rp, i32, vp, vp, sz, vp]
        lib.hs2_pages_copy.argtypes = [lp, rp, i32, vp, vp, i32, vp]
        for f in ("hs2_window_attn", "hs2_paged_attn_decode", "hs2_paged_attn_decode_fp8kv", "hs2_pages_reserve", "hs2_pages_write",
                  "hs2_pages_fork", "hs2_pages_free", "hs2_pages_compact", "hs2_pages_copy"):
            getattr(lib, f).restype = C.c_int
        for f in ("hs2_full_attn_select", "hs2_topk_select", "hs2_sparse_attn_prefill", "hs2_sparse_attn_decode",
                  "hs2_sparse_attn_prefill_gated", "hs2_sparse_attn_decode_gated", "hs2_sparse_attn_decode_static",
                  "hs2_sparse_attn_prefill_fp8kv", "hs2_sparse_attn_decode_fp8kv"):
            getattr(lib, f).restype = C.c_int
        _lib = lib
    return _lib


def hs2_device_error_flags() -> int:
    """Device error word of the library (0 = fine); synchronises the device."""
    v = C.c_uint(0)
    _check(load_library().hs2_device_error_flags(C.byref(v)), "hs2_device_error_flags")
    return int(v.value)


def hs2_set_filter_min_keys(min_keys: int) -> int:
    """Tuning knob: kv_len from which the full layer's selection uses filtered candidate lists; returns the old value."""
    return int(load_library().hs2_set_filter_min_keys(int(min_keys)))


def hs2_set_tcgen05_enabled(enabled: int) -> int:
    """Testing knob: 0 routes the full layer through its mma.sync kernels; returns the previous setting."""
    return int(load_library().hs2_set_tcgen05_enabled(int(enabled)))


def hs2_launch_count() -> int:
    """Kernels launched by the library in this process so far."""
    return int(load_library().hs2_launch_count())


def hs2_status_string(status: int) -> str:
    return load_library().hs2_status_string(int(status)).decode()


def _check(status: int, where: str):
    if status != HS2_OK:
        detail = ""
        if status == HS2_ERR_CUDA:
            detail = " (cudaError %d)" % load_library().hs2_last_cuda_error()
        raise HS2Error(status, where, detail)


def _dp(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream) -> C.c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def _axes(strides, rows: int):
    """``strides`` of a tensor of ``rows`` rows.  All of them 0 is `packed` to the library, which would read (or write) behind
    the one row of a tensor that is broadcast along every axis."""
    assert rows <= 1 or any(strides), "a tensor of one row, expanded: the library takes strides of 0 for packed"
    return strides


def _strides(t: torch.Tensor):
    assert t.stride(3) == 1, "last dimension must be contiguous"
    return (C.c_int64 * 3)(*_axes(t.stride()[:3], t.shape[:3].numel()))


def _scale_strides(t: torch.Tensor):
    return (C.c_int64 * 3)(*_axes(t.stride(), t.numel()))


class Problem:
    """Host-side description of one call; mirrors ``hs2_problem``."""

    def __init__(self, batch, q_len, kv_len, n_q_heads, n_kv_heads, head_dim, k_sel, window, dtype=torch.bfloat16,
                 softmax_scale: float = 0.0, q_start: Optional[torch.Tensor] = None,
                 kv_lens: Optional[torch.Tensor] = None, select_block: int = 0):
        self.batch, self.q_len, self.kv_len = int(batch), int(q_len), int(kv_len)
        self.n_q_heads, self.n_kv_heads, self.head_dim = int(n_q_heads), int(n_kv_heads), int(head_dim)
        self.k_sel, self.window = int(k_sel), int(window)
        self.dtype = dtype
        self.softmax_scale = float(softmax_scale)
        self.q_start, self.kv_lens = q_start, kv_lens
        self.select_block = int(select_block)
        for t in (q_start, kv_lens):
            assert t is None or (t.dtype == torch.int32 and t.is_cuda and t.is_contiguous())

    @classmethod
    def from_tensors(cls, q, k, k_sel, window, **kw):
        B, Lq, Hq, D = q.shape
        _, Lk, Hkv, _ = k.shape
        return cls(B, Lq, Lk, Hq, Hkv, D, k_sel, window, dtype=q.dtype, **kw)

    def c_struct(self, q=None, kv=None, o=None) -> _CProblem:
        if self.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("hs2 tensors are float32 or bfloat16")
        c = _CProblem(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.q_len, self.kv_len,
                      self.k_sel, self.window, self.softmax_scale,
                      HS2_F32 if self.dtype == torch.float32 else HS2_BF16,
                      None if self.q_start is None else self.q_start.data_ptr(),
                      None if self.kv_lens is None else self.kv_lens.data_ptr())
        c.select_block = self.select_block
        if q is not None:
            c.q_stride = _strides(q)
        if kv is not None:
            c.kv_stride = _strides(kv)
        if o is not None:
            c.o_stride = _strides(o)
        return c


def hs2_workspace_bytes(prob: Problem, op: int) -> int:
    c = prob.c_struct()
    return int(load_library().hs2_workspace_bytes(C.byref(c), int(op)))


def _workspace(prob: Problem, op: int, device, ws: Optional[torch.Tensor]):
    if ws is not None:
        return ws
    n = hs2_workspace_bytes(prob, op)
    return torch.empty(max(n, 256), dtype=torch.uint8, device=device)


def _check_inputs(prob: Problem, q, k, v):
    assert q.is_cuda and k.is_cuda and v.is_cuda, "hs2 runs on CUDA tensors only"
    assert q.dtype == k.dtype == v.dtype == prob.dtype
    assert tuple(q.shape) == (prob.batch, prob.q_len, prob.n_q_heads, prob.head_dim)
    assert tuple(k.shape) == tuple(v.shape) == (prob.batch, prob.kv_len, prob.n_kv_heads, prob.head_dim)
    assert k.stride() == v.stride(), "K and V share one stride triple"


def hs2_full_attn_select(prob: Problem, q, k, v, *, out=None, lse=None, idx=None, want_idx=True,
                         scores_dbg=None, want_scores=False, ws=None, stream=None):
    """FA layer: returns ``(O, LSE, idx | None, scores_dbg | None)``."""
    _check_inputs(prob, q, k, v)
    dev = q.device
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty(prob.batch, prob.n_q_heads, prob.q_len, dtype=torch.float32, device=dev) if lse is None else lse
    if idx is None and want_idx:
        idx = torch.empty(prob.batch, prob.n_kv_heads, prob.q_len, prob.k_sel, dtype=torch.int32, device=dev)
    if scores_dbg is None and want_scores:
        scores_dbg = torch.empty(prob.batch, prob.n_kv_heads, prob.q_len, prob.kv_len, dtype=torch.float32, device=dev)
    if idx is not None and scores_dbg is None:
        ws = _workspace(prob, HS2_OP_FULL_ATTN_SELECT, dev, ws)
    c = prob.c_struct(q, k, out)
    st = load_library().hs2_full_attn_select(C.byref(c), _dp(q), _dp(k), _dp(v), _dp(out), _dp(lse), _dp(idx),
                                             _dp(scores_dbg), _dp(ws), 0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "hs2_full_attn_select")
    return out, lse, idx, scores_dbg


def hs2_topk_select(prob: Problem, scores, *, idx=None, stream=None):
    """Token-level top-k outside the window on a float32 score tensor ``[B, Hkv, Lq, Lk]``."""
    assert scores.is_cuda and scores.dtype == torch.float32 and scores.is_contiguous()
    assert tuple(scores.shape) == (prob.batch, prob.n_kv_heads, prob.q_len, prob.kv_len)
    if idx is None:
        idx = torch.empty(prob.batch, prob.n_kv_heads, prob.q_len, prob.k_sel, dtype=torch.int32, device=scores.device)
    c = prob.c_struct()
    st = load_library().hs2_topk_select(C.byref(c), _dp(scores), _dp(idx), None, 0, _stream(stream))
    _check(st, "hs2_topk_select")
    return idx


def _sparse(fn_name, op, prob, q, k, v, idx, sink, out, lse, want_lse, ws, stream, gate=None):
    _check_inputs(prob, q, k, v)
    dev = q.device
    if idx is not None:
        assert idx.dtype == torch.int32 and idx.is_contiguous() and idx.is_cuda
        assert tuple(idx.shape) == (prob.batch, prob.n_kv_heads, prob.q_len, prob.k_sel)
    if sink is not None:
        assert sink.dtype == torch.float32 and sink.is_cuda and sink.numel() == prob.n_q_heads
    out = torch.empty_like(q) if out is None else out
    if lse is None and want_lse:
        lse = torch.empty(prob.batch, prob.n_q_heads, prob.q_len, dtype=torch.float32, device=dev)
    ws = _workspace(prob, op, dev, ws)
    c = prob.c_struct(q, k, out)
    if gate is not None:   # the gated entry point: gate logits laid out like the output
        assert gate.is_cuda and gate.dtype == out.dtype and gate.shape == out.shape and gate.stride() == out.stride()
        fn_name += "_gated"
        st = getattr(load_library(), fn_name)(C.byref(c), _dp(q), _dp(k), _dp(v), _dp(idx), _dp(sink), _dp(gate), _dp(out),
                                              _dp(lse), _dp(ws), ws.numel(), _stream(stream))
    else:
        st = getattr(load_library(), fn_name)(C.byref(c), _dp(q), _dp(k), _dp(v), _dp(idx), _dp(sink), _dp(out), _dp(lse),
                                              _dp(ws), ws.numel(), _stream(stream))
    _check(st, fn_name)
    return out, lse


def hs2_sparse_attn_prefill(prob: Problem, q, k, v, idx, *, sink=None, gate=None, out=None, lse=None, want_lse=False,
                            ws=None, stream=None):
    """SA layer, prefill: attention over (idx) U (forced window); returns ``(O, LSE | None)``.
    With ``gate`` (logits shaped like the output) the output is multiplied by sigmoid(gate) in the kernel's store."""
    return _sparse("hs2_sparse_attn_prefill", HS2_OP_SPARSE_ATTN_PREFILL, prob, q, k, v, idx, sink, out, lse,
                   want_lse, ws, stream, gate)


def hs2_sparse_attn_decode(prob: Problem, q, k, v, idx, *, sink=None, gate=None, out=None, lse=None, want_lse=False,
                           ws=None, stream=None):
    """SA layer, decode (q_len == 1, split over the attended set); returns ``(O, LSE | None)``."""
    return _sparse("hs2_sparse_attn_decode", HS2_OP_SPARSE_ATTN_DECODE, prob, q, k, v, idx, sink, out, lse,
                   want_lse, ws, stream, gate)


def _sparse_fp8(fn_name, prob, q, k8, v8, k_scale, v_scale, idx, sink, out, lse, want_lse, stream):
    assert q.is_cuda and q.dtype == torch.bfloat16 and q.stride(-1) == 1
    for t in (k8, v8):
        assert t.is_cuda and t.dtype == torch.uint8 and t.stride(-1) == 1
        assert tuple(t.shape) == (prob.batch, prob.kv_len, prob.n_kv_heads, prob.head_dim)
    assert k8.stride() == v8.stride()
    for t in (k_scale, v_scale):
        assert t.is_cuda and t.dtype == torch.float32
        assert tuple(t.shape) == (prob.batch, prob.kv_len, prob.n_kv_heads)
    assert k_scale.stride() == v_scale.stride()   # may be views into records that also hold the codes
    if idx is not None:
        assert idx.dtype == torch.int32 and idx.is_contiguous() and idx.is_cuda
        assert tuple(idx.shape) == (prob.batch, prob.n_kv_heads, prob.q_len, prob.k_sel)
    if sink is not None:
        assert sink.dtype == torch.float32 and sink.is_cuda and sink.numel() == prob.n_q_heads
    out = torch.empty_like(q) if out is None else out
    if lse is None and want_lse:
        lse = torch.empty(prob.batch, prob.n_q_heads, prob.q_len, dtype=torch.float32, device=q.device)
    c = prob.c_struct(q, k8, out)
    c.kv_scale_stride = _scale_strides(k_scale)
    st = getattr(load_library(), fn_name)(C.byref(c), _dp(q), _dp(k8), _dp(v8), _dp(k_scale), _dp(v_scale), _dp(idx),
                                          _dp(sink), _dp(out), _dp(lse), _stream(stream))
    _check(st, fn_name)
    return out, lse


def hs2_full_attn_select_fp8kv(prob: Problem, q, k8, v8, k_scale, v_scale, *, out=None, lse=None, idx=None, want_idx=True,
                               ws=None, stream=None):
    """FA layer, decode step (one query per sequence), on an e4m3 cache: returns ``(O, LSE, idx | None)``."""
    assert q.is_cuda and q.dtype == torch.bfloat16 and q.stride(-1) == 1
    for t in (k8, v8):
        assert t.is_cuda and t.dtype == torch.uint8 and t.stride(-1) == 1
        assert tuple(t.shape) == (prob.batch, prob.kv_len, prob.n_kv_heads, prob.head_dim)
    assert k8.stride() == v8.stride()
    for t in (k_scale, v_scale):
        assert t.is_cuda and t.dtype == torch.float32
        assert tuple(t.shape) == (prob.batch, prob.kv_len, prob.n_kv_heads)
    assert k_scale.stride() == v_scale.stride()   # may be views into records that also hold the codes
    dev = q.device
    out = torch.empty_like(q) if out is None else out
    lse = torch.empty(prob.batch, prob.n_q_heads, prob.q_len, dtype=torch.float32, device=dev) if lse is None else lse
    if idx is None and want_idx:
        idx = torch.empty(prob.batch, prob.n_kv_heads, prob.q_len, prob.k_sel, dtype=torch.int32, device=dev)
    if idx is not None:
        ws = _workspace(prob, HS2_OP_FULL_ATTN_SELECT_FP8KV, dev, ws)
    c = prob.c_struct(q, k8, out)
    c.kv_scale_stride = _scale_strides(k_scale)
    st = load_library().hs2_full_attn_select_fp8kv(C.byref(c), _dp(q), _dp(k8), _dp(v8), _dp(k_scale), _dp(v_scale), _dp(out),
                                                   _dp(lse), _dp(idx), _dp(ws), 0 if ws is None else ws.numel(), _stream(stream))
    _check(st, "hs2_full_attn_select_fp8kv")
    return out, lse, idx


def hs2_sparse_attn_prefill_fp8kv(prob: Problem, q, k8, v8, k_scale, v_scale, idx, *, sink=None, out=None, lse=None,
                                  want_lse=False, stream=None):
    """SA layer, prefill, on an e4m3 cache (uint8 codes + fp32 scale per (token, KV head)); bf16 Q and O."""
    return _sparse_fp8("hs2_sparse_attn_prefill_fp8kv", prob, q, k8, v8, k_scale, v_scale, idx, sink, out, lse, want_lse,
                       stream)


def hs2_sparse_attn_decode_fp8kv(prob: Problem, q, k8, v8, k_scale, v_scale, idx, *, sink=None, out=None, lse=None,
                                 want_lse=False, stream=None):
    """SA layer, decode (q_len == 1), on an e4m3 cache."""
    return _sparse_fp8("hs2_sparse_attn_decode_fp8kv", prob, q, k8, v8, k_scale, v_scale, idx, sink, out, lse, want_lse,
                       stream)


def hs2_kv_project(h, w, *, out=None, fp8=False, scales=None, stream=None):
    """Cache producer: ``out[T, N] = h[T, dm] @ w[N, dm].T`` (bf16), or with ``fp8=True`` e4m3 codes (uint8) plus one
    fp32 scale per (token, 128 columns).  ``out`` may be a strided 2-D view (e.g. a slice of a fused cache).
    Returns ``out`` or ``(out, scales)``."""
    assert h.is_cuda and w.is_cuda and h.dtype == torch.bfloat16 and w.dtype == torch.bfloat16
    assert h.dim() == 2 and w.dim() == 2 and h.shape[1] == w.shape[1] and h.stride(1) == 1 and w.stride(1) == 1
    T, dm = h.shape
    N = w.shape[0]
    if out is None:
        out = torch.empty(T, N, dtype=torch.uint8 if fp8 else torch.bfloat16, device=h.device)
    assert out.dim() == 2 and tuple(out.shape) == (T, N) and out.stride(1) == 1
    assert out.dtype == (torch.uint8 if fp8 else torch.bfloat16)
    if fp8 and scales is None:
        scales = torch.empty(T, N // 128, dtype=torch.float32, device=h.device)
    st = load_library().hs2_kv_project(T, dm, N, _dp(h), h.stride(0), _dp(w), w.stride(0), _dp(out), out.stride(0),
                                       _dp(scales) if fp8 else None, _stream(stream))
    _check(st, "hs2_kv_project")
    return (out, scales) if fp8 else out


def hs2_kv_project_fp8_records(h, w, codes, scales, *, stream=None):
    """Cache producer writing e4m3 codes and scales into records: ``codes`` is a uint8 view ``[T, G, 128]`` (G column
    groups = heads of dim 128, any 16-byte-multiple strides between tokens and groups, the 128 codes contiguous),
    ``scales`` a float32 view ``[T, G]``; both may point into the same buffer.  Returns ``(codes, scales)``."""
    assert h.is_cuda and w.is_cuda and h.dtype == torch.bfloat16 and w.dtype == torch.bfloat16
    assert h.dim() == 2 and w.dim() == 2 and h.shape[1] == w.shape[1] and h.stride(1) == 1 and w.stride(1) == 1
    T, dm = h.shape
    N = w.shape[0]
    assert codes.dtype == torch.uint8 and tuple(codes.shape) == (T, N // 128, 128) and codes.stride(2) == 1
    assert scales.dtype == torch.float32 and tuple(scales.shape) == (T, N // 128)
    st = load_library().hs2_kv_project_fp8_records(T, dm, N, _dp(h), h.stride(0), _dp(w), w.stride(0), _dp(codes),
                                                   codes.stride(0), codes.stride(1), _dp(scales), scales.stride(0),
                                                   scales.stride(1), _stream(stream))
    _check(st, "hs2_kv_project_fp8_records")
    return codes, scales


def hs2_probe_gather(prob: Problem, k, v, idx, *, mode=0, sink_word=None, stream=None):
    """Measurement aid: only the K/V row fetches of ``hs2_sparse_attn_prefill`` on this problem (same items, same
    order, same validity rules), no arithmetic.  ``mode`` 0 loads past L1, 1 through it.  Returns ``sink_word``."""
    assert k.is_cuda and v.is_cuda and k.dtype == torch.bfloat16
    if sink_word is None:
        sink_word = torch.zeros(1, dtype=torch.int32, device=k.device)
    c = prob.c_struct(None, k, None)
    st = load_library().hs2_probe_gather(C.byref(c), _dp(k), _dp(v), _dp(idx), int(mode), _dp(sink_word), _stream(stream))
    _check(st, "hs2_probe_gather")
    return sink_word


def hs2_sparse_attn_decode_static(prob: Problem, q, k, v, idx, *, sink=None, out, lse=None, stream=None):
    """Decode for callers that may not allocate: the split kernel's partials live in a fixed
    8.5 MB array inside the library, so no workspace is passed and nothing is allocated - here
    included, which is why ``out`` (and ``lse``, if wanted) must be given.  Limit:
    ``batch * n_kv_heads <= 64`` for groups of up to 8 query heads per KV head, ``<= 32`` for groups of 16 (which
    run as two sub-groups of 8).  Calls on one device share that array: keep them ordered on the GPU.
    """
    _check_inputs(prob, q, k, v)
    assert out is not None and out.is_cuda and out.shape == q.shape and out.dtype == q.dtype
    if idx is not None:
        assert idx.dtype == torch.int32 and idx.is_contiguous() and idx.is_cuda
    c = prob.c_struct(q, k, out)
    st = load_library().hs2_sparse_attn_decode_static(C.byref(c), _dp(q), _dp(k), _dp(v), _dp(idx), _dp(sink),
                                                      _dp(out), _dp(lse), _stream(stream))
    _check(st, "hs2_sparse_attn_decode_static")
    return out, lse


# The calls below are short enough on the GPU that what the host does counts: argument structs are packed in one go, and
# pointers and the stream travel as plain integers.
_PROBLEM = struct.Struct("@8i f i 2P 3q 3q 3q i 3q")
_PAGED = struct.Struct("@9i f i P q P 2q 2q 3q 3q")
_POOL = struct.Struct("@4i 3P")
_REGION = struct.Struct("@P 2i 3q")
assert _PROBLEM.size == C.sizeof(_CProblem) and _PAGED.size == C.sizeof(_CPagedProblem)
assert _POOL.size == C.sizeof(_CPagePool) and _REGION.size == C.sizeof(_CPageRegion)
_DTYPES = {torch.float32: HS2_F32, torch.bfloat16: HS2_BF16}
_ZERO3 = (0, 0, 0)
_current_stream = torch._C._cuda_getCurrentRawStream   # the handle alone: a Stream object costs 2 us


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _launch(name: str, device: torch.device, stream, *args):
    """Calls an entry point with `device` current and on its current stream (or the one given), and checks the status."""
    fn = getattr(load_library(), name)
    s = _current_stream(device.index) if stream is None else stream.cuda_stream
    if device.index == torch.cuda.current_device():
        st = fn(*args, s)
    else:
        with torch.cuda.device(device):
            st = fn(*args, s)
    if st:
        _check(st, name)


def _on_stream(fn):
    """A call with ``stream`` runs with that stream current: what it allocates (outputs, scratch) belongs to the stream then, and
    no later tensor of the caller's stream is put in its place while the kernels run."""
    @functools.wraps(fn)
    def call(*args, stream=None, **kw):
        if stream is None:
            return fn(*args, **kw)
        with torch.cuda.stream(stream):
            return fn(*args, stream=stream, **kw)
    return call


def _outputs(q, out, sink, gate, lse, want_lse, n_q_heads, lse_shape):
    """The output tensors, made where none were given (laid out like the gate, else like q), and the checks of what goes with
    them."""
    if out is None:
        out = torch.empty_like(q if gate is None else gate)
    else:
        assert out.device == q.device
        assert all(s or n == 1 for s, n in zip(out.stride(), out.shape)), "outputs of different rows share memory"
    if lse is None:
        if want_lse:
            lse = q.new_empty(lse_shape, dtype=torch.float32)
    else:
        assert lse.device == q.device and lse.dtype == torch.float32 and lse.is_contiguous() and tuple(lse.shape) == lse_shape
    if sink is not None:
        assert sink.dtype == torch.float32 and sink.device == q.device and sink.numel() == n_q_heads and sink.is_contiguous()
    assert out.dtype == q.dtype and out.shape == q.shape and out.stride(-1) == 1
    if gate is not None:   # gate logits laid out like the output
        assert gate.device == q.device and gate.dtype == out.dtype and gate.shape == out.shape and gate.stride() == out.stride()
    return out, lse


@_on_stream
def hs2_window_attn(prob: Problem, q, k, v, n_first: int = 0, *, sink=None, gate=None, out=None, lse=None, want_lse=False,
                    ws=None, stream=None):
    """Sliding-window layer: causal attention over the ``prob.window`` most recent tokens and the ``n_first`` first tokens
    of the sequence; ``sink`` and ``gate`` as in the sparse calls (``prob.k_sel`` does not matter, 0 will do).  Returns
    ``(O, LSE | None)``."""
    _check_inputs(prob, q, k, v)
    assert k.device == v.device == q.device
    B, L, Hq = prob.batch, prob.q_len, prob.n_q_heads
    out, lse = _outputs(q, out, sink, gate, lse, want_lse, Hq, (B, Hq, L))
    qs, ks, os_ = q.stride(), k.stride(), out.stride()
    assert qs[3] == ks[3] == 1, "last dimension must be contiguous"
    _axes(qs[:3], B * L * Hq)
    _axes(ks[:3], B * prob.kv_len * prob.n_kv_heads)
    c = _PROBLEM.pack(B, Hq, prob.n_kv_heads, prob.head_dim, L, prob.kv_len, prob.k_sel, prob.window, prob.softmax_scale,
                      _DTYPES[prob.dtype], _ptr(prob.q_start), _ptr(prob.kv_lens), *qs[:3], *ks[:3], *os_[:3], prob.select_block,
                      *_ZERO3)
    if L == 1 and ws is None:   # scratch for the keys that can be visible
        few = _CProblem.from_buffer_copy(c)
        few.kv_len = min(prob.kv_len, prob.window + max(0, n_first))
        n = load_library().hs2_workspace_bytes(C.byref(few), HS2_OP_WINDOW_ATTN)
        ws = q.new_empty(n, dtype=torch.uint8) if n else None
    _launch("hs2_window_attn", q.device, stream, c, n_first, q.data_ptr(), k.data_ptr(), v.data_ptr(), _ptr(sink), _ptr(gate),
            out.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel())
    return out, lse


class PagedProblem:
    """Host-side description of a paged decode call; mirrors ``hs2_paged_problem``.  ``window`` 0 is the whole context."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, page_size, n_pages, page_table, kv_lens, *, window: int = 0,
                 n_first: int = 0, dtype=torch.bfloat16, softmax_scale: float = 0.0):
        self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim = batch, n_q_heads, n_kv_heads, head_dim
        self.page_size, self.n_pages = page_size, n_pages
        self.window, self.n_first = window, n_first
        self.dtype, self.softmax_scale = dtype, softmax_scale
        if dtype not in _DTYPES:
            raise TypeError("hs2 tensors are float32 or bfloat16")
        rows, cols = page_table.shape
        stride = page_table.stride()
        assert page_table.dtype == kv_lens.dtype == torch.int32 and page_table.is_cuda and rows == batch
        assert stride[1] == 1 or cols == 1
        assert batch <= 1 or stride[0] >= cols, "the rows of the page table overlap: .contiguous() gives every sequence its own"
        assert kv_lens.is_contiguous() and tuple(kv_lens.shape) == (batch,) and kv_lens.device == page_table.device
        self.page_table, self.kv_lens = page_table, kv_lens
        self._cols, self._table_stride = cols, stride[0] if batch > 1 else max(stride[0], cols)

    @classmethod
    def from_tensors(cls, q, k_pages, page_table, kv_lens, **kw):
        B, _, Hq, D = q.shape
        n_pages, page_size, Hkv, _ = k_pages.shape
        return cls(B, Hq, Hkv, D, page_size, n_pages, page_table, kv_lens, dtype=q.dtype, **kw)

    def _pack(self, q=None, kv=None, o=None, scale=None) -> bytes:
        q, o = ((0, 0) if t is None else _axes(t.stride()[0:4:2], self.batch * self.n_q_heads) for t in (q, o))
        rows = self.n_pages * self.page_size * self.n_kv_heads
        kv, scale = (_ZERO3 if t is None else _axes(t.stride()[:3], rows) for t in (kv, scale))
        return _PAGED.pack(self.batch, self.n_q_heads, self.n_kv_heads, self.head_dim, self.page_size, self.n_pages, self._cols,
                           self.window, self.n_first, self.softmax_scale, _DTYPES[self.dtype], self.page_table.data_ptr(),
                           self._table_stride, self.kv_lens.data_ptr(), *q, *o, *kv, *scale)

    def c_struct(self, q=None, kv=None, o=None, scale=None) -> _CPagedProblem:
        return _CPagedProblem.from_buffer_copy(self._pack(q, kv, o, scale))


def hs2_paged_workspace_bytes(prob: PagedProblem) -> int:
    return int(load_library().hs2_paged_workspace_bytes(prob._pack()))


def _paged(name, prob: PagedProblem, q, k, v, scales, sink, gate, out, lse, want_lse, ws, stream):
    device, shape, strides = q.device, k.shape, k.stride()
    assert q.is_cuda and k.device == v.device == device == prob.page_table.device
    assert q.dtype == prob.dtype and q.shape == (prob.batch, 1, prob.n_q_heads, prob.head_dim) and q.stride(3) == 1
    assert shape == v.shape == (prob.n_pages, prob.page_size, prob.n_kv_heads, prob.head_dim)
    assert strides == v.stride() and strides[3] == 1, "K and V share one stride triple"
    if scales:
        assert k.dtype == v.dtype == torch.uint8
        for t in scales:
            assert t.device == device and t.dtype == torch.float32 and t.shape == shape[:3]
        assert scales[0].stride() == scales[1].stride()   # may be views into records that also hold the codes
    else:
        assert k.dtype == v.dtype == prob.dtype
    out, lse = _outputs(q, out, sink, gate, lse, want_lse, prob.n_q_heads, (prob.batch, prob.n_q_heads, 1))
    c = prob._pack(q, k, out, scales[0] if scales else None)
    if ws is None:
        n = load_library().hs2_paged_workspace_bytes(c)
        ws = q.new_empty(n, dtype=torch.uint8) if n else None
    _launch(name, device, stream, c, q.data_ptr(), k.data_ptr(), v.data_ptr(), *[t.data_ptr() for t in scales], _ptr(sink),
            _ptr(gate), out.data_ptr(), _ptr(lse), _ptr(ws), 0 if ws is None else ws.numel())
    return out, lse


@_on_stream
def hs2_paged_attn_decode(prob: PagedProblem, q, k_pages, v_pages, *, sink=None, gate=None, out=None, lse=None, want_lse=False,
                          ws=None, stream=None):
    """Attention of one new token per sequence (``q [B, 1, Hq, D]``) over a cache in pages (``[n_pages, page_size, Hkv, D]``);
    returns ``(O, LSE | None)``."""
    return _paged("hs2_paged_attn_decode", prob, q, k_pages, v_pages, (), sink, gate, out, lse, want_lse, ws, stream)


@_on_stream
def hs2_paged_attn_decode_fp8kv(prob: PagedProblem, q, k8_pages, v8_pages, k_scale, v_scale, *, sink=None, gate=None, out=None,
                                lse=None, want_lse=False, ws=None, stream=None):
    """The same on an e4m3 cache (uint8 codes + fp32 scale per (token, KV head), ``[n_pages, page_size, Hkv]``); bf16 Q, O."""
    return _paged("hs2_paged_attn_decode_fp8kv", prob, q, k8_pages, v8_pages, (k_scale, v_scale), sink, gate, out, lse, want_lse,
                  ws, stream)


class PagePool:
    """Who owns which page; mirrors ``hs2_page_pool``.  ``ref_counts [n_pages]``, ``page_table [max_seqs, max_pages]`` and
    ``lens [max_seqs]`` are int32 tensors that the calls change in place; ``PagePool.empty`` makes those of an empty pool."""

    def __init__(self, page_size: int, ref_counts, page_table, lens):
        self.device = ref_counts.device
        for t in (ref_counts, page_table, lens):
            assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.device == self.device
        (n_pages,), (rows, cols) = ref_counts.shape, page_table.shape
        assert lens.shape == (rows,)
        self.page_size, self.n_pages = page_size, n_pages
        self.ref_counts, self.page_table, self.lens = ref_counts, page_table, lens
        self._packed = _POOL.pack(n_pages, page_size, rows, cols, ref_counts.data_ptr(), page_table.data_ptr(), lens.data_ptr())

    @classmethod
    def empty(cls, n_pages: int, page_size: int, max_seqs: int, max_pages: int, device="cuda"):
        new = lambda shape, fill: torch.full(shape, fill, dtype=torch.int32, device=device)  # noqa: E731
        return cls(page_size, new((n_pages,), 0), new((max_seqs, max_pages), -1), new((max_seqs,), 0))

    def c_struct(self) -> _CPagePool:
        return _CPagePool.from_buffer_copy(self._packed)

    def _list(self, t, n=None):
        """The pointer and the length of an int32 list on the pool's device."""
        assert t.dtype == torch.int32 and t.device == self.device and t.dim() == 1 and t.is_contiguous()
        assert n is None or t.shape[0] == n
        return t.data_ptr(), t.shape[0]


def _dense(shape, strides):
    """Elements of a block with these axes, which has to be contiguous."""
    n = 1
    for size, stride in zip(reversed(shape), reversed(strides)):
        assert size == 1 or stride == n, "the bytes of a token are contiguous"
        n *= size
    return n


def _regions(pool: PagePool, tensors):
    """``[n_pages, page_size, ...]`` or, for several layers, ``[layers, n_pages, page_size, ...]`` tensors as packed structs,
    and for each the number of axes before the pages."""
    assert len(tensors) <= HS2_MAX_PAGE_REGIONS
    lead, packed, axes = (pool.n_pages, pool.page_size), b"", []
    for t in tensors:
        shape, strides, size = t.shape, t.stride(), t.element_size()
        one, many = shape[:2] == lead, shape[1:3] == lead
        if one == many:
            raise ValueError("a region is [n_pages, page_size, ...] or [layers, n_pages, page_size, ...]; got %s" % (tuple(shape),))
        assert t.device == pool.device
        at = 1 if many else 0
        row = _dense(shape[at + 2:], strides[at + 2:]) * size
        token = strides[at + 1] * size if lead[1] > 1 else row   # the stride of an axis of one element means nothing
        page = strides[at] * size if lead[0] > 1 else max(strides[at] * size, lead[1] * token)
        packed += _REGION.pack(t.data_ptr(), shape[0] if many else 1, row, strides[0] * size if many else 0, page, token)
        axes.append(at)
    return packed or None, axes


def _pages_ws(pool, n, ws):
    if ws is None:
        ws = pool.ref_counts.new_empty(load_library().hs2_pages_workspace_bytes(pool._packed, n), dtype=torch.uint8)
    return ws.data_ptr(), ws.numel()


def hs2_pages_workspace_bytes(pool: PagePool, n: int) -> int:
    return int(load_library().hs2_pages_workspace_bytes(pool._packed, int(n)))


@_on_stream
def hs2_pages_reserve(pool: PagePool, regions, seqs, n_new, *, start=None, ws=None, stream=None):
    """Room for ``n_new[i]`` more tokens of sequence ``seqs[i]`` (a shared, partly filled last page is copied in every
    region); returns ``start``: the position of the first new token, -1 where the request was refused."""
    ps, n = pool._list(seqs)
    pn, _ = pool._list(n_new, n)
    start = torch.empty_like(seqs) if start is None else start
    _launch("hs2_pages_reserve", pool.device, stream, pool._packed, _regions(pool, regions)[0], len(regions), ps, pn, n,
            pool._list(start, n)[0], *_pages_ws(pool, n, ws))
    return start


@_on_stream
def hs2_pages_write(pool: PagePool, regions, rows, seqs, start, n_new, *, stream=None):
    """Writes ``rows[r] [n, T, ...]`` (``[layers, n, T, ...]`` for a region with layers): row ``t < n_new[i]`` of request ``i``
    goes to position ``start[i] + t`` of sequence ``seqs[i]``."""
    ps, n = pool._list(seqs)
    (pt, _), (pn, _) = pool._list(start, n), pool._list(n_new, n)
    assert len(rows) == len(regions)
    packed, axes = _regions(pool, regions)
    pointers, strides, max_new = [], [], None
    for t, at, region in zip(rows, axes, regions):
        shape, st, size = t.shape, t.stride(), t.element_size()
        assert t.device == pool.device and t.dtype == region.dtype and shape[at + 2:] == region.shape[at + 2:]
        assert shape[at] == n and (not at or shape[0] == region.shape[0]) and max_new in (None, shape[at + 1])
        _dense(shape[at + 2:], st[at + 2:])
        max_new = shape[at + 1]
        pointers.append(t.data_ptr())
        strides += (st[0] * size if at else 0, st[at] * size, st[at + 1] * size)
    if max_new and n:
        _launch("hs2_pages_write", pool.device, stream, pool._packed, packed, len(regions), struct.pack("@%dP" % len(rows), *pointers),
                struct.pack("@%dq" % len(strides), *strides), ps, pt, pn, n, max_new)


@_on_stream
def hs2_pages_fork(pool: PagePool, src, dst, *, ws=None, stream=None):
    """Sequence ``dst[i]`` becomes what ``src[i]`` was before the call and shares its pages; all at once."""
    ps, n = pool._list(src)
    _launch("hs2_pages_fork", pool.device, stream, pool._packed, ps, pool._list(dst, n)[0], n, *_pages_ws(pool, n, ws))


@_on_stream
def hs2_pages_free(pool: PagePool, seqs, keep=None, *, stream=None):
    """Sequence ``seqs[i]`` keeps its first ``keep[i]`` tokens (none without ``keep``) and gives its other pages back."""
    ps, n = pool._list(seqs)
    _launch("hs2_pages_free", pool.device, stream, pool._packed, ps, None if keep is None else pool._list(keep, n)[0], n)


@_on_stream
def hs2_pages_compact(pool: PagePool, regions, *, moved=None, ws=None, stream=None):
    """Moves the pages in use to the low end of the pool; returns ``moved [n_pages]``: the new index of every page that was
    in use, -1 for the others."""
    moved = torch.empty_like(pool.ref_counts) if moved is None else moved
    _launch("hs2_pages_compact", pool.device, stream, pool._packed, _regions(pool, regions)[0], len(regions),
            pool._list(moved, pool.n_pages)[0], *_pages_ws(pool, 0, ws))
    return moved


@_on_stream
def hs2_pages_copy(pool: PagePool, regions, src, dst, *, stream=None):
    """Copies the contents of page ``src[i]`` to page ``dst[i]`` in every region; no bookkeeping."""
    ps, n = pool._list(src)
    _launch("hs2_pages_copy", pool.device, stream, pool._packed, _regions(pool, regions)[0], len(regions), ps, pool._list(dst, n)[0], n)
