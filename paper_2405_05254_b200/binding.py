"""Thin ctypes binding of the C-ABI library (argument marshalling only).

Function names mirror ``include/yoco_xattn.h``.  Tensors are torch CUDA tensors (torch is used
for device memory and streams only); lengths and offsets are host numpy int32 arrays.  There is
no fallback: if the CUDA library has not been built, every call raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libyoco_xattn.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE_TOO_SMALL, ERR_CUDA, ERR_TIMEOUT = 0, -1, -2, -3, -4, -5
ERR_STATIC_SCRATCH_EXCEEDED = -6
ERR_BAD_PAGE, ERR_HOST_MEMORY = -7, -8
MODE_DECODE, MODE_CHUNK = 0, 1


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("d", ctypes.c_int32), ("T", ctypes.c_int32), ("scale", ctypes.c_float),
                ("kv_head_stride", ctypes.c_int64), ("max_kv_len", ctypes.c_int32),
                ("window", ctypes.c_int32)]


class KvAppendShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("T", ctypes.c_int32),
                ("d_model", ctypes.c_int32), ("eps", ctypes.c_float), ("kv_head_stride", ctypes.c_int64)]


class PagedLayout(ctypes.Structure):
    _fields_ = [("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("table_stride", ctypes.c_int32),
                ("rope_pairs", ctypes.c_int32), ("page_rows", ctypes.c_int64), ("cos_sin", ctypes.c_void_p),
                ("max_pos", ctypes.c_int32)]


class PagedAppendShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("d", ctypes.c_int32), ("T", ctypes.c_int32),
                ("src_stride", ctypes.c_int64)]


class GretShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("T", ctypes.c_int32),
                ("num_slots", ctypes.c_int32), ("scale", ctypes.c_float), ("tau", ctypes.c_float), ("decay_bf16", ctypes.c_int32),
                ("q_stride", ctypes.c_int64), ("k_stride", ctypes.c_int64), ("v_stride", ctypes.c_int64),
                ("o_stride", ctypes.c_int64), ("decay_stride", ctypes.c_int64)]


class NormGate(ctypes.Structure):
    _fields_ = [("gate", ctypes.c_void_p), ("gain", ctypes.c_void_p), ("bias", ctypes.c_void_p),
                ("gate_stride", ctypes.c_int64), ("eps", ctypes.c_float), ("rms", ctypes.c_int32)]


class HeadNormShape(ctypes.Structure):
    _fields_ = [("tokens", ctypes.c_int64), ("H", ctypes.c_int32), ("d", ctypes.c_int32), ("x_stride", ctypes.c_int64),
                ("y_stride", ctypes.c_int64)]


class RopeShape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hk", ctypes.c_int32), ("d", ctypes.c_int32),
                ("T", ctypes.c_int32), ("rot", ctypes.c_int32), ("rope_pairs", ctypes.c_int32), ("q_stride", ctypes.c_int64),
                ("k_stride", ctypes.c_int64), ("q_out_stride", ctypes.c_int64), ("k_out_stride", ctypes.c_int64)]


class Segment(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("group", "b", "c", "k_begin", "k_end", "slot")]


class PlanInfo(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("mode", "tile_n", "tile_m", "m_tiles", "num_groups", "num_ctas", "num_streams",
                 "num_segments", "max_splits", "needs_combine")] + \
               [("total_tiles", ctypes.c_int64), ("workspace_bytes", ctypes.c_int64),
                ("sub_items", ctypes.c_int32), ("num_slots", ctypes.c_int32)]


class YocoError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        msg = lib().yoco_xattn_strerror(code).decode()
        if code == ERR_CUDA:
            msg += f" [cudaError {lib().yoco_xattn_last_cuda_error()}]"
        super().__init__(f"{where}: {msg} ({code})")


_lib = None


def lib() -> ctypes.CDLL:
    """Load libyoco_xattn.so; fails loudly when it is missing (there is no CPU path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with paper_2405_05254_b200.build.build_cuda_library()")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        L.yoco_xattn_plan.argtypes = [ctypes.POINTER(Shape), vp, i32, i32, ctypes.POINTER(PlanInfo), vp, i32]
        L.yoco_xattn_workspace_size.argtypes = [ctypes.POINTER(Shape), vp, i32, i32, ctypes.POINTER(sz)]
        run_args = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.yoco_xattn_decode.argtypes = run_args
        L.yoco_xattn_chunk.argtypes = run_args
        L.yoco_xattn_decode_static.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, vp]
        L.yoco_xattn_static_scratch_bytes.argtypes = []
        L.yoco_xattn_combine.argtypes = [i64, i32, i32, vp, vp, vp, vp, vp]
        L.yoco_xattn_combine_gathered.argtypes = [i64, i32, i32, vp, vp, vp, vp, vp]
        L.yoco_xattn_decode_partial.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        part_at = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.yoco_xattn_decode_partial_at.argtypes = part_at
        L.yoco_xattn_chunk_partial_at.argtypes = part_at
        L.yoco_xattn_workspace_size_at.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, i32, i32, ctypes.POINTER(sz)]
        L.yoco_xattn_plan_at.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, i32, i32, ctypes.POINTER(PlanInfo), vp, i32]
        for name in ("yoco_xattn_decode_partial_at", "yoco_xattn_chunk_partial_at", "yoco_xattn_workspace_size_at",
                     "yoco_xattn_plan_at"):
            getattr(L, name).restype = i32
        L.yoco_xattn_decode_fp8.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, sz, vp]
        L.yoco_xattn_decode_fp8.restype = i32
        L.yoco_xattn_chunk_fp8.argtypes = L.yoco_xattn_decode_fp8.argtypes
        L.yoco_xattn_chunk_fp8.restype = i32
        L.yoco_xattn_workspace_size_chunk_fp8.argtypes = [ctypes.POINTER(Shape), vp, i32, ctypes.POINTER(sz)]
        L.yoco_xattn_workspace_size_chunk_fp8.restype = i32
        L.yoco_kv_fold_gain.argtypes = [i64, i64, vp, vp, vp, vp]
        L.yoco_kv_append.argtypes = [ctypes.POINTER(KvAppendShape), vp, vp, vp, vp, vp, vp, vp, vp]
        L.yoco_xattn_sub_bound.argtypes = [ctypes.c_int64, i32, i32]
        L.yoco_xattn_sub_bound.restype = ctypes.c_int64
        L.yoco_kv_append_fp8.argtypes = [ctypes.POINTER(KvAppendShape), vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.yoco_kv_append_fp8.restype = i32
        L.yoco_kv_append_status.argtypes = [vp]
        for name in ("yoco_kv_fold_gain", "yoco_kv_append", "yoco_kv_append_status"):
            getattr(L, name).restype = i32
        L.yoco_xattn_status.argtypes = [vp, vp]
        L.yoco_xattn_status_detail.argtypes = [vp, vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.yoco_xattn_decode_status_word.argtypes = [i32, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.yoco_kv_append_status_detail.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i32)]
        L.yoco_xattn_selftest_wait_expiry.argtypes = [ctypes.POINTER(Shape), vp, vp, vp, vp, vp, vp, vp, sz, i32, vp]
        for name in ("yoco_xattn_status_detail", "yoco_xattn_decode_status_word", "yoco_kv_append_status_detail",
                     "yoco_xattn_selftest_wait_expiry"):
            getattr(L, name).restype = i32
        lay = ctypes.POINTER(PagedLayout)
        rows = [ctypes.POINTER(PagedAppendShape), lay]
        L.yoco_xattn_workspace_size_paged.argtypes = [ctypes.POINTER(Shape), lay, vp, i32, i32, i32, ctypes.POINTER(sz)]
        attend, attend_q4 = [vp] * 7 + [vp, sz, vp], [vp] * 9 + [vp, sz, vp]
        for name, args in (("yoco_xattn_decode_paged", [ctypes.POINTER(Shape), lay] + attend),
                           ("yoco_xattn_chunk_paged", [ctypes.POINTER(Shape), lay] + attend),
                           ("yoco_xattn_decode_paged_q4", [ctypes.POINTER(Shape), lay] + attend_q4),
                           ("yoco_xattn_chunk_paged_q4", [ctypes.POINTER(Shape), lay] + attend_q4),
                           ("yoco_paged_append", rows + [vp] * 8), ("yoco_paged_append_q4", rows + [vp] * 10),
                           ("yoco_paged_gather", rows + [vp] * 8), ("yoco_paged_gather_q4", rows + [vp] * 10),
                           ("yoco_rope_q", [ctypes.POINTER(Shape), lay] + [vp] * 4),
                           ("yoco_xattn_selftest_wait_expiry_paged", [ctypes.POINTER(Shape), lay] + [vp] * 9 + [sz, i32, vp])):
            getattr(L, name).argtypes = args
            getattr(L, name).restype = i32
        L.yoco_xattn_workspace_size_paged.restype = i32
        L.yoco_xattn_workspace_bound_paged.argtypes = L.yoco_xattn_workspace_size_paged.argtypes
        L.yoco_xattn_workspace_bound_paged.restype = i32
        for name, args in (("yoco_gret_step", [vp] * 11), ("yoco_gret_chunk", [vp] * 12 + [sz, vp]),
                           ("yoco_gret_workspace_size", [vp, vp, i32, ctypes.POINTER(sz)]),
                           ("yoco_gret_workspace_bound", [vp, vp, i32, ctypes.POINTER(sz)]),
                           ("yoco_gret_selftest_wait_expiry", [vp] * 12 + [sz, i32, vp]),
                           ("yoco_head_norm", [vp] * 5), ("yoco_rope", [vp] * 9)):
            getattr(L, name).argtypes = args
            getattr(L, name).restype = i32
        L.yoco_xattn_profile_enable.argtypes = [i32]
        L.yoco_xattn_profile_collect.argtypes = [vp, i32, vp]
        L.yoco_xattn_strerror.argtypes = [i32]
        L.yoco_xattn_strerror.restype = ctypes.c_char_p
        L.yoco_xattn_last_cuda_error.argtypes = []
        for name in ("plan", "workspace_size", "decode", "chunk", "combine", "status", "last_cuda_error",
                     "profile_enable", "profile_collect", "decode_static", "static_scratch_bytes",
                     "combine_gathered", "decode_partial"):
            getattr(L, "yoco_xattn_" + name).restype = i32
        _lib = L
    return _lib


def make_shape(B, Hq, Hkv, d, T, scale=0.0, kv_head_stride=0, max_kv_len=0, window=0) -> Shape:
    """``window`` = C > 0 selects the sliding-window mask (row i sees i - C < j <= i); 0 = none."""
    return Shape(B, Hq, Hkv, d, T, float(scale), int(kv_head_stride), int(max_kv_len), int(window))


def _host_i32(a):
    if a is None:
        return None, None
    arr = np.ascontiguousarray(a, dtype=np.int32)
    return arr, ctypes.c_void_p(arr.ctypes.data)


def yoco_xattn_plan(shape: Shape, kv_len, sm_count: int, mode: int):
    """Returns (PlanInfo, list of Segment) of the split/tile heuristic; host only."""
    keep, p_len = _host_i32(kv_len)
    info = PlanInfo()
    rc = lib().yoco_xattn_plan(ctypes.byref(shape), p_len, sm_count, mode, ctypes.byref(info), None, 0)
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_plan")
    segs = (Segment * max(1, info.num_segments))()
    rc = lib().yoco_xattn_plan(ctypes.byref(shape), p_len, sm_count, mode, ctypes.byref(info),
                               ctypes.cast(segs, ctypes.c_void_p), info.num_segments)
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_plan")
    return info, list(segs)[: info.num_segments]


def yoco_xattn_plan_at(shape: Shape, kv_len, key_offset, kv_total, sm_count: int, mode: int):
    """(PlanInfo, segments) for one key shard at a given place in the whole sequences; host only."""
    keep, p_len = _host_i32(kv_len)
    keep_off, p_off = _host_i32(key_offset)
    keep_tot, p_tot = _host_i32(kv_total)
    info = PlanInfo()
    rc = lib().yoco_xattn_plan_at(ctypes.byref(shape), p_len, p_off, p_tot, sm_count, mode, ctypes.byref(info), None, 0)
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_plan_at")
    segs = (Segment * max(1, info.num_segments))()
    rc = lib().yoco_xattn_plan_at(ctypes.byref(shape), p_len, p_off, p_tot, sm_count, mode, ctypes.byref(info),
                                  ctypes.cast(segs, ctypes.c_void_p), info.num_segments)
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_plan_at")
    return info, list(segs)[: info.num_segments]


def yoco_xattn_workspace_size(shape: Shape, kv_len, mode: int, sm_count: int = 0) -> int:
    keep, p_len = _host_i32(kv_len)
    out = ctypes.c_size_t(0)
    rc = lib().yoco_xattn_workspace_size(ctypes.byref(shape), p_len, sm_count, mode, ctypes.byref(out))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_workspace_size")
    return int(out.value)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


def _stream_ptr(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _run(fn_name, shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream):
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    fn = getattr(lib(), fn_name)
    rc = fn(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len, _ptr(O), _ptr(lse),
            _ptr(workspace), workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, fn_name)


def yoco_xattn_decode(shape: Shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream=None) -> None:
    """Enqueue split-KV decode attention (G*T <= 16 rows per KV head) on the stream."""
    _run("yoco_xattn_decode", shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream)


class PreparedCall:
    """A decode or chunk call whose arguments are marshalled once: a serving loop that makes the same
    layer call every step (same buffers, same lengths) pays the ctypes conversions a single time.
    The tensors and arrays are kept alive by the object; run() only enqueues."""

    def __init__(self, fn_name, shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream=None):
        self._keep = (shape, Q, K, V, O, lse, workspace, stream) + _host_i32(cu_kv)[:1] + _host_i32(kv_len)[:1]
        p_cu = None if self._keep[-2] is None else ctypes.c_void_p(self._keep[-2].ctypes.data)
        p_len = None if self._keep[-1] is None else ctypes.c_void_p(self._keep[-1].ctypes.data)
        self._name = fn_name
        self._fn = getattr(lib(), fn_name)
        self._args = (ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len, _ptr(O), _ptr(lse), _ptr(workspace),
                      ctypes.c_size_t(workspace.numel() * workspace.element_size()), _stream_ptr(stream))

    def run(self) -> None:
        rc = self._fn(*self._args)
        if rc != OK:
            raise YocoError(rc, self._name)


def prepare_decode(shape: Shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream=None) -> PreparedCall:
    """yoco_xattn_decode with its arguments marshalled once; call .run() to enqueue it."""
    return PreparedCall("yoco_xattn_decode", shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream)


def yoco_xattn_chunk(shape: Shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream=None) -> None:
    """Enqueue the multi-token (tcgen05) attention on the stream."""
    _run("yoco_xattn_chunk", shape, Q, K, V, cu_kv, kv_len, O, lse, workspace, stream)


def yoco_xattn_combine(part_o, part_lse, O, lse=None, stream=None) -> None:
    """Merge partials: part_o [rows,S,d] fp32, part_lse [rows,S] fp32 -> O [rows,d] bf16."""
    rows, S, d = part_o.shape
    rc = lib().yoco_xattn_combine(rows, S, d, _ptr(part_o), _ptr(part_lse), _ptr(O), _ptr(lse),
                                  _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_combine")


def yoco_xattn_combine_gathered(part_o, part_lse, O, lse=None, stream=None) -> None:
    """Merge piece-major partials: part_o [S,rows,d] fp32, part_lse [S,rows] fp32 -> O [rows,d] bf16."""
    S, rows, d = part_o.shape
    rc = lib().yoco_xattn_combine_gathered(rows, S, d, _ptr(part_o), _ptr(part_lse), _ptr(O), _ptr(lse),
                                           _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_combine_gathered")


def yoco_xattn_decode_partial(shape: Shape, Q, K, V, cu_kv, kv_len, part_o, part_lse, workspace,
                              stream=None) -> None:
    """Decode over the key shard this GPU holds: fp32 partial rows + their log-sum-exp (T = 1)."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    rc = lib().yoco_xattn_decode_partial(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len,
                                         _ptr(part_o), _ptr(part_lse), _ptr(workspace),
                                         workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_decode_partial")


def yoco_xattn_partial_at(shape: Shape, Q, K, V, cu_kv, kv_len, key_offset, kv_total, part_o, part_lse, workspace,
                          mode: int = MODE_DECODE, stream=None) -> None:
    """One key shard's partial result with the shard's place in the whole sequences (host int32 [B] each:
    first key held here, length of the whole sequence): any T and any window.  ``mode`` picks the split-KV
    decode kernel (G*T <= 16) or the tensor-core chunk kernel."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    keep_off, p_off = _host_i32(key_offset)
    keep_tot, p_tot = _host_i32(kv_total)
    name = "yoco_xattn_decode_partial_at" if mode == MODE_DECODE else "yoco_xattn_chunk_partial_at"
    rc = getattr(lib(), name)(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len, p_off, p_tot,
                              _ptr(part_o), _ptr(part_lse), _ptr(workspace),
                              workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, name)


def yoco_xattn_workspace_size_at(shape: Shape, kv_len, key_offset, kv_total, mode: int, sm_count: int = 0) -> int:
    keep_len, p_len = _host_i32(kv_len)
    keep_off, p_off = _host_i32(key_offset)
    keep_tot, p_tot = _host_i32(kv_total)
    out = ctypes.c_size_t(0)
    rc = lib().yoco_xattn_workspace_size_at(ctypes.byref(shape), p_len, p_off, p_tot, sm_count, mode, ctypes.byref(out))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_workspace_size_at")
    return int(out.value)


def yoco_xattn_decode_fp8(shape: Shape, Q, K8, V8, k_scale, v_scale, cu_kv, kv_len, O, lse, workspace,
                          stream=None) -> None:
    """Decode over an FP8 E4M3 cache (uint8 device tensors) with per-head scales (host float32 [Hkv])."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    ks = np.ascontiguousarray(k_scale, dtype=np.float32)
    vs = np.ascontiguousarray(v_scale, dtype=np.float32)
    rc = lib().yoco_xattn_decode_fp8(ctypes.byref(shape), _ptr(Q), _ptr(K8), _ptr(V8),
                                     ctypes.c_void_p(ks.ctypes.data), ctypes.c_void_p(vs.ctypes.data), p_cu, p_len,
                                     _ptr(O), _ptr(lse), _ptr(workspace),
                                     workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_decode_fp8")


def yoco_xattn_chunk_fp8(shape: Shape, Q, K8, V8, k_scale, v_scale, cu_kv, kv_len, O, lse, workspace,
                         stream=None) -> None:
    """The multi-token (tensor-core) path over an FP8 E4M3 cache with per-head scales; any T."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    ks = np.ascontiguousarray(k_scale, dtype=np.float32)
    vs = np.ascontiguousarray(v_scale, dtype=np.float32)
    rc = lib().yoco_xattn_chunk_fp8(ctypes.byref(shape), _ptr(Q), _ptr(K8), _ptr(V8),
                                    ctypes.c_void_p(ks.ctypes.data), ctypes.c_void_p(vs.ctypes.data), p_cu, p_len,
                                    _ptr(O), _ptr(lse), _ptr(workspace),
                                    workspace.numel() * workspace.element_size(), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_chunk_fp8")


def yoco_xattn_workspace_size_chunk_fp8(shape: Shape, kv_len, sm_count: int = 0) -> int:
    keep, p_len = _host_i32(kv_len)
    out = ctypes.c_size_t(0)
    rc = lib().yoco_xattn_workspace_size_chunk_fp8(ctypes.byref(shape), p_len, sm_count, ctypes.byref(out))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_workspace_size_chunk_fp8")
    return int(out.value)


def yoco_kv_fold_gain(g, W, Wg, stream=None) -> None:
    """Wg = g[:, None] * W rounded to bf16 (W, Wg: [d_model, n_out] bf16 device tensors)."""
    d_model, n_out = W.shape
    rc = lib().yoco_kv_fold_gain(d_model, n_out, _ptr(g), _ptr(W), _ptr(Wg), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_kv_fold_gain")


def yoco_kv_append(shape: KvAppendShape, X, Wgk, Wgv, K, V, cu_kv, kv_len, stream=None) -> None:
    """Enqueue K^ = RMSNorm(X) W_K, V^ = RMSNorm(X) W_V and store the rows at the last T positions
    of every sequence in the packed caches K, V (in place)."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    rc = lib().yoco_kv_append(ctypes.byref(shape), _ptr(X), _ptr(Wgk), _ptr(Wgv), _ptr(K), _ptr(V), p_cu, p_len,
                              _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_kv_append")


def yoco_xattn_sub_bound(n_tiles: int, sub_items: int, r: int) -> int:
    return int(lib().yoco_xattn_sub_bound(n_tiles, sub_items, r))


def yoco_kv_append_fp8(shape: KvAppendShape, X, Wgk, Wgv, K8, V8, k_scale, v_scale, cu_kv, kv_len, stream=None) -> None:
    """As yoco_kv_append, but the rows are stored as FP8 E4M3 bytes (uint8 caches) after division by the
    per-head scales (host float32 [Hkv])."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    ks = np.ascontiguousarray(k_scale, dtype=np.float32)
    vs = np.ascontiguousarray(v_scale, dtype=np.float32)
    rc = lib().yoco_kv_append_fp8(ctypes.byref(shape), _ptr(X), _ptr(Wgk), _ptr(Wgv), _ptr(K8), _ptr(V8),
                                  ctypes.c_void_p(ks.ctypes.data), ctypes.c_void_p(vs.ctypes.data), p_cu, p_len,
                                  _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_kv_append_fp8")


def yoco_kv_append_status(stream=None) -> int:
    """Synchronise the stream; 0 unless an append kernel gave up a bounded wait since the last call."""
    return int(lib().yoco_kv_append_status(_stream_ptr(stream)))


def yoco_xattn_status(workspace, stream=None) -> int:
    """Synchronise the stream and return the status of the last call that used ``workspace`` (0 = ok);
    ``workspace=None`` reads the built-in buffer of yoco_xattn_decode_static on the current device."""
    return int(lib().yoco_xattn_status(_ptr(workspace), _stream_ptr(stream)))


STATUS_BAD_PAGE = 7
WAIT_ITEM_QUEUE, WAIT_RING_FULL, WAIT_RING_EMPTY, WAIT_TENSOR, WAIT_DRAIN, WAIT_MISALIGNED = 1, 2, 3, 4, 5, 6


def yoco_xattn_status_detail(workspace, stream=None):
    """(status, wait_class, cta): which kind of bounded wait ran out first, and in which CTA."""
    wc, cta = ctypes.c_int32(0), ctypes.c_int32(0)
    rc = lib().yoco_xattn_status_detail(_ptr(workspace), _stream_ptr(stream), ctypes.byref(wc), ctypes.byref(cta))
    return int(rc), int(wc.value), int(cta.value)


def yoco_xattn_decode_status_word(word: int):
    """Pure host: (status, wait_class, cta) of a status word."""
    wc, cta = ctypes.c_int32(0), ctypes.c_int32(0)
    rc = lib().yoco_xattn_decode_status_word(int(word), ctypes.byref(wc), ctypes.byref(cta))
    return int(rc), int(wc.value), int(cta.value)


def yoco_kv_append_status_detail(stream=None):
    wc, cta = ctypes.c_int32(0), ctypes.c_int32(0)
    rc = lib().yoco_kv_append_status_detail(_stream_ptr(stream), ctypes.byref(wc), ctypes.byref(cta))
    return int(rc), int(wc.value), int(cta.value)


def yoco_xattn_selftest_wait_expiry(shape: Shape, Q, K, V, cu_kv, kv_len, O, workspace, limit_ms: int, stream=None) -> None:
    """Run the decode kernel with a producer that starts no copy and a wait limit of ``limit_ms``: the
    first tile wait runs out, the kernel records it and returns.  O is left undefined."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    rc = lib().yoco_xattn_selftest_wait_expiry(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len, _ptr(O),
                                               _ptr(workspace), workspace.numel() * workspace.element_size(),
                                               int(limit_ms), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_selftest_wait_expiry")


def yoco_xattn_selftest_wait_expiry_fp8(shape: Shape, Q, K8, V8, k_scale, v_scale, cu_kv, kv_len, O, workspace,
                                        limit_ms: int, stream=None) -> None:
    """The same self-test for the decode kernel of the 8-bit cache: the wait that runs out is the consumers'
    wait for the producer to arm their tile.  O is left undefined."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    ks = np.ascontiguousarray(k_scale, dtype=np.float32)
    vs = np.ascontiguousarray(v_scale, dtype=np.float32)
    rc = lib().yoco_xattn_selftest_wait_expiry_fp8(ctypes.byref(shape), _ptr(Q), _ptr(K8), _ptr(V8),
                                                   ctypes.c_void_p(ks.ctypes.data), ctypes.c_void_p(vs.ctypes.data),
                                                   p_cu, p_len, _ptr(O), _ptr(workspace),
                                                   workspace.numel() * workspace.element_size(), int(limit_ms),
                                                   _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_selftest_wait_expiry_fp8")


def yoco_xattn_selftest_wait_expiry_paged(shape: Shape, layout: PagedLayout, Q, pools, page_table, kv_len, O, workspace,
                                          limit_ms: int, stream=None) -> None:
    """The same self-test over a paged cache; ``pools``: (K, V) of a bf16 cache, (K4, K_scale, V4, V_scale) of a 4-bit one.  O
    is left undefined."""
    keep_len, p_len = _host_i32(kv_len)
    K, Ks, V, Vs = pools if len(pools) == 4 else (pools[0], None, pools[1], None)
    rc = lib().yoco_xattn_selftest_wait_expiry_paged(
        ctypes.byref(shape), ctypes.byref(layout), _ptr(Q), _ptr(K), _ptr(Ks), _ptr(V), _ptr(Vs), _ptr(page_table), p_len, _ptr(O),
        _ptr(workspace), workspace.numel() * workspace.element_size(), int(limit_ms), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_selftest_wait_expiry_paged")


# ---- paged cache -----------------------------------------------------------------------------------
def make_paged_layout(page_size, num_pages, table_stride, page_rows=0, cos_sin=None, rope_pairs=0) -> PagedLayout:
    """``cos_sin``: fp32 CUDA tensor [positions, d] (d/2 cosines, then d/2 sines) or None; it is kept alive by the layout."""
    if cos_sin is not None and (str(cos_sin.dtype) != "torch.float32" or cos_sin.dim() != 2 or not cos_sin.is_contiguous()):
        raise ValueError("cos_sin must be a contiguous fp32 tensor [positions, d]")
    layout = PagedLayout(int(page_size), int(num_pages), int(table_stride), int(rope_pairs), int(page_rows),
                         None if cos_sin is None else cos_sin.data_ptr(), 0 if cos_sin is None else cos_sin.shape[0])
    layout.tensor = cos_sin
    return layout


# What each argument after (shape, layout) is: "q" bf16 rows [B, Hq, T, d], "g" bf16 output of a gather, "x" bf16 rows of
# the new tokens (strided between tokens), "k" bf16 pool, "c" pool of 4-bit codes, "s" pool of their scales, "i" device
# table of pages, "n" host int32 array or None, "l" fp32 [B, Hq, T] or None, "w" workspace bytes.
_PAGED_ARGS = {
    "yoco_xattn_decode_paged": "qkkinqlw", "yoco_xattn_chunk_paged": "qkkinqlw",
    "yoco_xattn_decode_paged_q4": "qcscsinqlw", "yoco_xattn_chunk_paged_q4": "qcscsinqlw",
    "yoco_paged_append": "xxkkinn", "yoco_paged_append_q4": "xxcscsinn",
    "yoco_paged_gather": "kkinngg", "yoco_paged_gather_q4": "cscsinngg",
    "yoco_rope_q": "qnq",
}
_PAGED_TYPES = {"q": "torch.bfloat16", "g": "torch.bfloat16", "x": "torch.bfloat16", "k": "torch.bfloat16", "c": "torch.uint8",
                "s": "torch.float16", "i": "torch.int32", "l": "torch.float32"}


class PreparedPagedCall:
    """A call of one of the paged-cache functions whose arguments are checked and marshalled once; run() only
    enqueues, on ``stream`` or, without one, on the stream that is current then.  The tensors are kept alive; shape, layout
    and the numbers of rows (``new_len``, ``begin``, ``end``) are copied.  ``kv_len``, if a contiguous int32 array, is read
    at every run(), so a serving loop may advance its lengths in place; its workspace is then sized by
    yoco_xattn_workspace_bound_paged with the lengths that it will reach."""

    def __init__(self, fn_name, shape, layout, *args, stream=None):
        import torch
        kinds = _PAGED_ARGS[fn_name]
        if len(args) != len(kinds):
            raise TypeError(f"{fn_name} takes {len(kinds)} arguments after the layout, got {len(args)}")
        self._keep = [layout, stream]
        shape, cos_sin = type(shape).from_buffer_copy(shape), getattr(layout, "tensor", None)
        layout = PagedLayout.from_buffer_copy(layout)
        self._keep += [shape, layout]
        out, device, host = [ctypes.addressof(shape), ctypes.addressof(layout)], torch.cuda.current_device(), []
        for n, (kind, a) in enumerate(zip(kinds, args)):
            if kind == "n":
                lengths = kinds == "qnq" or "w" in kinds or ("x" in kinds and n == len(kinds) - 1)      # kv_len
                keep = _host_i32(a if lengths or a is None else np.array(a, dtype=np.int32))[0]
                if keep is not None and keep.size < shape.B:
                    raise ValueError(f"{fn_name}: host array {n} has {keep.size} entries for {shape.B} sequences")
                self._keep.append(keep)
                host.append(keep)
                out.append(None if keep is None else keep.ctypes.data)
                continue
            if a is None and kind == "l":
                out.append(None)
                continue
            if not a.is_cuda or a.device.index != device:
                raise ValueError(f"{fn_name}: tensor {n} is on {a.device}, the current device is cuda:{device}")
            if str(a.dtype) != _PAGED_TYPES.get(kind, str(a.dtype)):
                raise ValueError(f"{fn_name}: tensor {n} has type {a.dtype}, not {_PAGED_TYPES[kind]}")
            if not self._in_order(kind, a, shape, layout):
                raise ValueError(f"{fn_name}: tensor {n} has strides {a.stride()}, which are not those of the call")
            self._keep.append(a)
            out.append(a.data_ptr())
            if kind == "w":
                out.append(a.numel() * a.element_size())
        if cos_sin is not None and (cos_sin.shape[1] != shape.d or cos_sin.device != torch.device("cuda", device)):
            raise ValueError(f"{fn_name}: cos_sin is {tuple(cos_sin.shape)} on {cos_sin.device} for head dimension {shape.d}")
        self._check_sizes(fn_name, kinds, shape, layout, args, host)
        self._stream = None if stream is None else stream.cuda_stream
        self._current_stream, self._device = torch._C._cuda_getCurrentRawStream, device
        self._others = torch.cuda.device_count() > 1
        # every argument is a pointer or a size: a prototype of integers costs 0.2 us less a call than pointer objects
        proto = ctypes.CFUNCTYPE(ctypes.c_int32, *[ctypes.c_void_p] * (len(out) + 1))
        self._name, self._fn, self._args = fn_name, proto((fn_name, lib())), tuple(out)

    @staticmethod
    def _in_order(kind, a, shape, layout):
        """Whether the tensor's strides are those that the call goes by: contiguous, or rows (of all heads of a token, of a
        page, of a sequence's table) that lie src_stride, page_rows or table_stride apart.  Rows that are
        contiguous, but wider or narrower than that, are not; a tensor without a dimension for the rows lies as the caller says.
        (A pool's dimension may count parts of the distance between pages, K and V pages in turn say: it is held to its size.)"""
        if a.numel() == 0:
            return True
        elems = {"k": shape.d, "c": shape.d // 2, "s": shape.d // 32}.get(kind)
        if kind == "x":
            width, apart = shape.Hkv * shape.d, shape.src_stride or shape.Hkv * shape.d
        elif kind == "i":
            width, apart = a.shape[-1] if a.dim() else 1, layout.table_stride
        elif elems:
            width = shape.Hkv * layout.page_size * elems
            apart = layout.page_rows * elems or width
        else:
            return a.is_contiguous()
        n, i = 1, a.dim()
        while i > 0 and n < width:                 # the dimensions of one row, densely
            i -= 1
            if a.shape[i] != 1 and a.stride(i) != n:
                return False
            n *= a.shape[i]
        # dimensions between a row and the next one: K and V pages side by side, or a token's K, V and more, in one tensor
        while i > 1 and n < apart and a.stride(i - 1) == n and n * a.shape[i - 1] <= apart:
            i -= 1
            n *= a.shape[i]
        if elems and i > 0 and apart % n == 0 and a.is_contiguous():
            return True
        for j in reversed(range(i)):               # the rows, `apart` from one another
            if a.shape[j] != 1 and a.stride(j) != apart:
                return False
            apart *= a.shape[j]
        return True

    @staticmethod
    def _check_sizes(fn_name, kinds, shape, layout, args, host):
        """Every tensor holds what the call may touch (elements from its first one to the end of its storage)."""
        P, B = layout.page_size, shape.B
        rows = (layout.num_pages - 1) * (layout.page_rows or shape.Hkv * P) + shape.Hkv * P
        need = {"i": B * layout.table_stride, "k": rows * shape.d, "c": rows * (shape.d // 2), "s": rows * (shape.d // 32)}
        if "q" in kinds:
            need["l"] = B * shape.Hq * shape.T
            need["q"] = need["l"] * shape.d
        elif "x" in kinds:
            tokens = int(host[0][:B].sum()) if host[0] is not None else B * shape.T
            need["x"] = max(0, tokens - 1) * (shape.src_stride or shape.Hkv * shape.d) + shape.Hkv * shape.d if tokens else 0
        elif host[0] is not None and host[1] is not None:
            need["g"] = int((host[1][:B].astype(np.int64) - host[0][:B]).sum()) * shape.Hkv * shape.d
        for n, (kind, a) in enumerate(zip(kinds, args)):
            if a is not None and kind in need:
                have = a.untyped_storage().nbytes() // a.element_size() - a.storage_offset()
                if have < need[kind]:
                    raise ValueError(f"{fn_name}: tensor {n} holds {have} elements, the call needs {need[kind]}")

    def run(self) -> None:
        if self._others:
            import torch
            if torch.cuda.current_device() != self._device:
                raise ValueError(f"{self._name}: prepared for cuda:{self._device}, the current device is cuda:{torch.cuda.current_device()}")
        stream = self._stream
        rc = self._fn(*self._args, self._current_stream(self._device) if stream is None else stream)
        if rc != OK:
            raise YocoError(rc, self._name)


def prepare_paged(fn_name, shape, layout, *args, stream=None) -> PreparedPagedCall:
    """``fn_name(shape, layout, *args)`` with its arguments marshalled once; call .run() to enqueue it."""
    return PreparedPagedCall(fn_name, shape, layout, *args, stream=stream)


def _workspace_paged(name, shape, layout, kv_len, mode, q4, sm_count):
    keep, p_len = _host_i32(kv_len)
    out = ctypes.c_size_t(0)
    rc = getattr(lib(), name)(ctypes.byref(shape), ctypes.byref(layout), p_len, sm_count, mode, int(q4), ctypes.byref(out))
    if rc != OK:
        raise YocoError(rc, name)
    return int(out.value)


def yoco_xattn_workspace_size_paged(shape: Shape, layout: PagedLayout, kv_len, mode: int, q4: bool = False,
                                    sm_count: int = 0) -> int:
    """Workspace bytes for exactly these lengths."""
    return _workspace_paged("yoco_xattn_workspace_size_paged", shape, layout, kv_len, mode, q4, sm_count)


def yoco_xattn_workspace_bound_paged(shape: Shape, layout: PagedLayout, kv_len, mode: int, q4: bool = False,
                                     sm_count: int = 0) -> int:
    """Workspace bytes that suffice for all lengths up to these: for a workspace kept while the sequences grow."""
    return _workspace_paged("yoco_xattn_workspace_bound_paged", shape, layout, kv_len, mode, q4, sm_count)


def yoco_xattn_decode_paged(shape: Shape, layout: PagedLayout, Q, K_pages, V_pages, page_table, kv_len, O, lse, workspace,
                            stream=None) -> None:
    """Enqueue attention of a few query rows (G*T <= 16) over a paged bf16 cache."""
    prepare_paged("yoco_xattn_decode_paged", shape, layout, Q, K_pages, V_pages, page_table, kv_len, O, lse, workspace,
                  stream=stream).run()


def yoco_xattn_decode_paged_q4(shape: Shape, layout: PagedLayout, Q, K4, K_scale, V4, V_scale, page_table, kv_len, O, lse,
                               workspace, stream=None) -> None:
    """The same over 4-bit pages (codes [pages, Hkv, P, d/2] bytes, scales [pages, Hkv, P, d/32] fp16)."""
    prepare_paged("yoco_xattn_decode_paged_q4", shape, layout, Q, K4, K_scale, V4, V_scale, page_table, kv_len, O, lse,
                  workspace, stream=stream).run()


def yoco_xattn_chunk_paged(shape: Shape, layout: PagedLayout, Q, K_pages, V_pages, page_table, kv_len, O, lse, workspace,
                           stream=None) -> None:
    """Enqueue the multi-token (tcgen05) attention over a paged bf16 cache; any T."""
    prepare_paged("yoco_xattn_chunk_paged", shape, layout, Q, K_pages, V_pages, page_table, kv_len, O, lse, workspace,
                  stream=stream).run()


def yoco_xattn_chunk_paged_q4(shape: Shape, layout: PagedLayout, Q, K4, K_scale, V4, V_scale, page_table, kv_len, O, lse,
                              workspace, stream=None) -> None:
    """The multi-token attention over 4-bit pages; any T."""
    prepare_paged("yoco_xattn_chunk_paged_q4", shape, layout, Q, K4, K_scale, V4, V_scale, page_table, kv_len, O, lse,
                  workspace, stream=stream).run()


def yoco_paged_append(shape: PagedAppendShape, layout: PagedLayout, K_new, V_new, K_pages, V_pages, page_table, new_len,
                      kv_len, stream=None) -> None:
    """Store the new tokens' rows (keys turned by their positions when the layout has a table) in the last
    ``new_len[i]`` (None: T) positions of every sequence."""
    prepare_paged("yoco_paged_append", shape, layout, K_new, V_new, K_pages, V_pages, page_table, new_len, kv_len,
                  stream=stream).run()


def yoco_paged_append_q4(shape: PagedAppendShape, layout: PagedLayout, K_new, V_new, K4, K_scale, V4, V_scale, page_table,
                         new_len, kv_len, stream=None) -> None:
    """The same into 4-bit pages."""
    prepare_paged("yoco_paged_append_q4", shape, layout, K_new, V_new, K4, K_scale, V4, V_scale, page_table, new_len,
                  kv_len, stream=stream).run()


def yoco_paged_gather(shape: PagedAppendShape, layout: PagedLayout, K_pages, V_pages, page_table, begin, end, K, V,
                      stream=None) -> None:
    """Read positions [begin[i], end[i]) back as a packed head-major bf16 cache."""
    prepare_paged("yoco_paged_gather", shape, layout, K_pages, V_pages, page_table, begin, end, K, V, stream=stream).run()


def yoco_paged_gather_q4(shape: PagedAppendShape, layout: PagedLayout, K4, K_scale, V4, V_scale, page_table, begin, end, K,
                         V, stream=None) -> None:
    """The same from 4-bit pages: the values they stand for, rounded to bf16."""
    prepare_paged("yoco_paged_gather_q4", shape, layout, K4, K_scale, V4, V_scale, page_table, begin, end, K, V,
                  stream=stream).run()


def yoco_rope_q(shape: Shape, layout: PagedLayout, Q, kv_len, Q_rot, stream=None) -> None:
    """Turn the queries [B, Hq, T, d] by the angles of their rows' positions N_i - T + t."""
    prepare_paged("yoco_rope_q", shape, layout, Q, kv_len, Q_rot, stream=stream).run()


# ---- self-decoder: token-major rows -------------------------------------------------------------------
def make_gret_shape(B, H, d, T=1, num_slots=0, scale=0.0, tau=0.0, decay_bf16=False, q_stride=0, k_stride=0, v_stride=0,
                    o_stride=0, decay_stride=0) -> GretShape:
    """``tau`` > 0: the decays are logits z of g = sigmoid(z)^(1/tau); 0: natural logarithms of g.  ``num_slots`` 0: B."""
    return GretShape(int(B), int(H), int(d), int(T), int(num_slots) or int(B), float(scale), float(tau), int(decay_bf16),
                     int(q_stride), int(k_stride), int(v_stride), int(o_stride), int(decay_stride))


def make_norm_gate(eps, rms=False, gate=None, gain=None, bias=None, gate_stride=None) -> NormGate:
    """Normalisation of the heads' outputs, gain, bias (bf16 [H * d] or None) and gate (bf16 rows or None; ``gate_stride`` None:
    the distance of the tensor's tokens).  The tensors are kept alive by the object."""
    if gate_stride is None:
        gate_stride = gate.stride(0) if gate is not None and gate.dim() > 1 and gate.shape[0] > 1 else 0
    norm = NormGate(None if gate is None else gate.data_ptr(), None if gain is None else gain.data_ptr(),
                    None if bias is None else bias.data_ptr(), int(gate_stride), float(eps), int(rms))
    norm.tensors = {"gate": gate, "gain": gain, "bias": bias}
    return norm


def make_rope_shape(B, Hq, Hk, d, T=1, rot=0, pairs=0, q_stride=0, k_stride=0, q_out_stride=0, k_out_stride=0) -> RopeShape:
    """``rot``: channels of a head that turn (0: all); ``pairs``: 0 halves, 1 neighbours."""
    return RopeShape(int(B), int(Hq), int(Hk), int(d), int(T), int(rot), int(pairs), int(q_stride), int(k_stride),
                     int(q_out_stride), int(k_out_stride))


# The arguments after the shape: rows (bf16, named by their stride in the shape), "decay", "norm" (NormGate or None), "state", "freq" (fp64
# [rot / 2]), host int32 arrays [B] or None ("slots", "pos": read at every run; "lens": copied), "workspace" bytes.
_TOKEN_ARGS = {
    "yoco_gret_step": ("q", "k", "v", "decay", "norm", "state", "slots", "slots", "o"),
    "yoco_gret_chunk": ("q", "k", "v", "decay", "norm", "state", "slots", "slots", "lens", "o", "workspace"),
    "yoco_head_norm": ("x", "norm", "y"),
    "yoco_rope": ("q", "k", "freq", "pos", "lens", "q_out", "k_out"),
}


_token_fns = {}


def _rows_lie(a, width: int, apart: int) -> bool:
    """Whether the tensor's strides are those of rows of ``width`` elements, ``apart`` from one another (a tensor without
    a dimension for the rows lies as the caller says)."""
    n, i = 1, a.dim()
    while i > 0 and n < width:                     # the dimensions of one row, densely
        i -= 1
        if a.shape[i] != 1 and a.stride(i) != n:
            return False
        n *= a.shape[i]
    for j in reversed(range(i)):
        if a.shape[j] != 1 and a.stride(j) != apart:
            return False
        apart *= a.shape[j]
    return True


class PreparedTokensCall:
    """A call over token-major rows whose arguments are checked and marshalled once; run() only enqueues, on ``stream`` or, without
    one, on the stream that is current then.  The tensors are kept alive; shape and lengths are copied.  Slots and positions, if contiguous
    int32 arrays, are read at every run(), so a serving loop may change them in place."""

    def __init__(self, fn_name, shape, *args, stream=None):
        import torch
        kinds = _TOKEN_ARGS[fn_name]
        if len(args) != len(kinds):
            raise TypeError(f"{fn_name} takes {len(kinds)} arguments after the shape, got {len(args)}")
        shape = type(shape).from_buffer_copy(shape)
        device = torch.cuda.current_device()
        self._keep, out = [shape, stream], [ctypes.addressof(shape)]
        lens = args[kinds.index("lens")] if "lens" in kinds else None
        if lens is not None:
            lens = np.array(lens, dtype=np.int32)
            if lens.size < shape.B:
                raise ValueError(f"{fn_name}: {lens.size} lengths for {shape.B} sequences")
        if fn_name == "yoco_head_norm":
            tokens = shape.tokens
        elif "lens" in kinds:
            tokens = shape.B * shape.T if lens is None else int(lens[:shape.B].sum(dtype=np.int64))
        else:
            tokens = shape.B
        rope = fn_name == "yoco_rope"

        def device_tensor(name, a, dtype, elements, width=0, apart=0):
            if not a.is_cuda or a.device.index != device:
                raise ValueError(f"{fn_name}: {name} is on {a.device}, the current device is cuda:{device}")
            if dtype is not None and a.dtype != dtype:
                raise ValueError(f"{fn_name}: {name} has type {a.dtype}, not {dtype}")
            if a.numel() and not (_rows_lie(a, width, apart) if width else a.is_contiguous()):
                raise ValueError(f"{fn_name}: {name} has strides {a.stride()}, which are not those of the call")
            have = a.untyped_storage().nbytes() // a.element_size() - a.storage_offset()
            if have < elements:
                raise ValueError(f"{fn_name}: {name} holds {have} elements, the call needs {elements}")
            self._keep.append(a)

        def rows(name, a, width, stride, dtype=torch.bfloat16):
            apart = stride or width
            device_tensor(name, a, dtype, (tokens - 1) * apart + width if tokens > 0 else 0, width, apart)

        for kind, a in zip(kinds, args):
            if kind in ("slots", "pos", "lens"):
                keep = lens if kind == "lens" else _host_i32(a)[0]
                if keep is not None and keep.size < shape.B:
                    raise ValueError(f"{fn_name}: a host array has {keep.size} entries for {shape.B} sequences")
                self._keep.append(keep)
                out.append(None if keep is None else keep.ctypes.data)
                continue
            if kind == "norm":
                norm = None if a is None else NormGate.from_buffer_copy(a)
                if norm is not None:
                    for name, t in getattr(a, "tensors", {}).items():
                        if t is not None and name == "gate":
                            rows(name, t, shape.H * shape.d, norm.gate_stride)
                        elif t is not None:
                            device_tensor(name, t, torch.bfloat16, shape.H * shape.d)
                self._keep.append(norm)
                out.append(None if norm is None else ctypes.addressof(norm))
                continue
            if a is None:
                if not (kind == "workspace" or (rope and kind in ("k", "k_out") and shape.Hk == 0)):
                    raise ValueError(f"{fn_name}: {kind} is missing")
                out += [None, 0] if kind == "workspace" else [None]
                continue
            if kind == "decay":
                rows(kind, a, shape.H, shape.decay_stride, torch.bfloat16 if shape.decay_bf16 else torch.float32)
            elif kind == "state":
                device_tensor(kind, a, torch.float32, shape.num_slots * shape.H * shape.d * shape.d)
            elif kind == "freq":
                device_tensor(kind, a, torch.float64, (shape.rot or shape.d) // 2)
            elif kind == "workspace":
                device_tensor(kind, a, None, 0)
            else:
                heads = (shape.Hk if kind in ("k", "k_out") else shape.Hq) if rope else shape.H
                rows(kind, a, heads * shape.d, getattr(shape, kind + "_stride"))
            out.append(a.data_ptr())
            if kind == "workspace":
                out.append(a.numel() * a.element_size())
        self._stream = None if stream is None else stream.cuda_stream
        self._current_stream, self._device = torch._C._cuda_getCurrentRawStream, device
        self._others = torch.cuda.device_count() > 1
        if fn_name not in _token_fns:              # integers as arguments, see PreparedPagedCall
            _token_fns[fn_name] = ctypes.CFUNCTYPE(ctypes.c_int32, *[ctypes.c_void_p] * (len(out) + 1))((fn_name, lib()))
        self._name, self._fn, self._args = fn_name, _token_fns[fn_name], tuple(out)

    def run(self) -> None:
        if self._others:
            import torch
            if torch.cuda.current_device() != self._device:
                raise ValueError(f"{self._name}: prepared for cuda:{self._device}, the current device is cuda:{torch.cuda.current_device()}")
        stream = self._stream
        rc = self._fn(*self._args, self._current_stream(self._device) if stream is None else stream)
        if rc != OK:
            raise YocoError(rc, self._name)


def prepare_tokens(fn_name, shape, *args, stream=None) -> PreparedTokensCall:
    """``fn_name(shape, *args)`` with its arguments marshalled once; call .run() to enqueue it."""
    return PreparedTokensCall(fn_name, shape, *args, stream=stream)


def _gret_workspace(fn_name, shape, lens, sm_count) -> int:
    keep, p_len = _host_i32(lens)
    if keep is not None and keep.size < shape.B:
        raise ValueError(f"{fn_name}: {keep.size} lengths for {shape.B} sequences")
    out = ctypes.c_size_t(0)
    rc = getattr(lib(), fn_name)(ctypes.byref(shape), p_len, sm_count, ctypes.byref(out))
    if rc != OK:
        raise YocoError(rc, fn_name)
    return int(out.value)


def yoco_gret_workspace_size(shape: GretShape, lens=None, sm_count: int = 0) -> int:
    """Workspace bytes of yoco_gret_chunk for exactly these lengths (None: shape.T each); may be 0."""
    return _gret_workspace("yoco_gret_workspace_size", shape, lens, sm_count)


def yoco_gret_workspace_bound(shape: GretShape, lens=None, sm_count: int = 0) -> int:
    """Workspace bytes that suffice for all lengths up to these: for a workspace kept while sequences come and go."""
    return _gret_workspace("yoco_gret_workspace_bound", shape, lens, sm_count)


def yoco_gret_chunk(shape: GretShape, Q, K, V, decay, norm, state, slot_in, slot_out, lens, O, workspace=None, stream=None) -> None:
    """Enqueue gated retention over whole prompts or chunks of them: ``lens`` [B] tokens (None: shape.T each), states from slots
    ``slot_in`` (-1: zero) into slots ``slot_out`` (-1: not kept; None: slot i of sequence i)."""
    prepare_tokens("yoco_gret_chunk", shape, Q, K, V, decay, norm, state, slot_in, slot_out, lens, O, workspace, stream=stream).run()


def yoco_gret_selftest_wait_expiry(shape: GretShape, Q, K, V, decay, norm, state, slot_in, slot_out, lens, O, workspace, limit_ms: int,
                                   stream=None) -> None:
    """Self-test of the bounded waits (arguments as for yoco_gret_chunk): a producer that starts no copy and a limit of ``limit_ms``.  O and the
    slots that the call writes are left undefined."""
    call = prepare_tokens("yoco_gret_chunk", shape, Q, K, V, decay, norm, state, slot_in, slot_out, lens, O, workspace)
    rc = lib().yoco_gret_selftest_wait_expiry(*call._args, int(limit_ms), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_gret_selftest_wait_expiry")


def yoco_gret_step(shape: GretShape, Q, K, V, decay, norm, state, slot_in, slot_out, O, stream=None) -> None:
    """The same for one token of every sequence."""
    prepare_tokens("yoco_gret_step", shape, Q, K, V, decay, norm, state, slot_in, slot_out, O, stream=stream).run()


def yoco_head_norm(shape: HeadNormShape, X, norm: NormGate, Y, stream=None) -> None:
    """Normalise every head's channels, gain, bias, swish gate; Y may be X."""
    prepare_tokens("yoco_head_norm", shape, X, norm, Y, stream=stream).run()


def yoco_rope(shape: RopeShape, Q, K, inv_freq, pos, lens, Q_rot, K_rot, stream=None) -> None:
    """Turn queries and keys (None with Hk = 0) by the angles of their positions pos[i], pos[i] + 1, ..."""
    prepare_tokens("yoco_rope", shape, Q, K, inv_freq, pos, lens, Q_rot, K_rot, stream=stream).run()


def yoco_xattn_profile_enable(max_records: int) -> None:
    rc = lib().yoco_xattn_profile_enable(max_records)
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_profile_enable")


def yoco_xattn_profile_collect(capacity: int) -> np.ndarray:
    """Durations (ms) of the attention kernel of the calls recorded since the last collect."""
    buf = np.zeros(max(1, capacity), dtype=np.float32)
    n = ctypes.c_int32(0)
    rc = lib().yoco_xattn_profile_collect(ctypes.c_void_p(buf.ctypes.data), capacity, ctypes.byref(n))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_profile_collect")
    return buf[: n.value].copy()


def yoco_xattn_decode_static(shape: Shape, Q, K, V, cu_kv, kv_len, O, lse, stream=None) -> None:
    """Decode for callers that cannot allocate: same result as yoco_xattn_decode, but the split
    tables and partial results live in a 4 MiB buffer built into the library instead of a
    caller-provided workspace.  Raises YocoError(ERR_STATIC_SCRATCH_EXCEEDED) when the problem
    needs more than that.  Calls that may overlap on the GPU must not both use this entry."""
    keep_cu, p_cu = _host_i32(cu_kv)
    keep_len, p_len = _host_i32(kv_len)
    rc = lib().yoco_xattn_decode_static(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), p_cu, p_len,
                                        _ptr(O), _ptr(lse), _stream_ptr(stream))
    if rc != OK:
        raise YocoError(rc, "yoco_xattn_decode_static")


def yoco_xattn_static_scratch_bytes() -> int:
    return int(lib().yoco_xattn_static_scratch_bytes())
