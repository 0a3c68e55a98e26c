"""Thin ctypes binding of libqp_hip.so: argument marshalling only.

Every function has the name and argument order of its C-ABI counterpart in include/qp.h
(the path), include/qp_layer.h (the decoder layer around it) or include/qp_paged.h (the paged cache) and takes torch tensors on the GPU (device memory and streams are all torch is used for).
There is no CPU fallback: if the library is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional

import torch

from .build import LIB_PATH

QP_OK, QP_ERR_INVALID_ARG, QP_ERR_UNSUPPORTED, QP_ERR_CAPACITY, QP_ERR_HIP = range(5)
QP_F32, QP_BF16 = 0, 1
QP_SCORE_KEY_NORM_SMALL, QP_SCORE_VALUE_NORM, QP_SCORE_WINDOW_ATTN = 0, 1, 2
QP_ATTEND_AUTO, QP_ATTEND_SCALAR, QP_ATTEND_MFMA, QP_ATTEND_MFMA_DECODE = 0, 1, 2, 3
QP_SCORE_WINDOW_LOGIT, QP_SCORE_SHARED_HEADS = 3, 0x100
RULES = {"key_norm_small": QP_SCORE_KEY_NORM_SMALL, "value_norm": QP_SCORE_VALUE_NORM,
         "window_attn": QP_SCORE_WINDOW_ATTN, "window_logit": QP_SCORE_WINDOW_LOGIT}
RULES.update({name + "+shared": code | QP_SCORE_SHARED_HEADS for name, code in list(RULES.items())})
QP_MAX_GROUP_TOKENS = 32768


class qp_layout(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("dtype", ctypes.c_int32), ("softmax_scale", ctypes.c_float)]


class qp_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("capacity", ctypes.c_int32), ("len", ctypes.c_int32), ("format", ctypes.c_int32)]


QP_CACHE_SAME, QP_CACHE_FP8_E4M3 = 0, 1


class qp_attend_plan_info(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("workgroups", ctypes.c_int32), ("key_chunks", ctypes.c_int32),
                ("tiles_per_chunk", ctypes.c_int32), ("mirrored_rows", ctypes.c_int32),
                ("scratch_bytes", ctypes.c_size_t), ("split_row_blocks", ctypes.c_int32)]


class qp_layer_shape(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int32), ("d_ff", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_theta", ctypes.c_float), ("mrope_section", ctypes.c_int32 * 3)]


class qp_layer_weights(ctypes.Structure):
    _fields_ = [(name, ctypes.c_void_p) for name in
                ("ln1_w", "w_qkv", "b_qkv", "w_o", "ln2_w", "w_gate_up", "w_down")]


class qp_paged_cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("pos", ctypes.c_void_p), ("weight", ctypes.c_void_p),
                ("n_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32), ("format", ctypes.c_int32)]


class qp_paged_batch(ctypes.Structure):
    _fields_ = [("page_table", ctypes.c_void_p), ("len", ctypes.c_void_p), ("row_start", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("table_pages", ctypes.c_int32), ("n_rows", ctypes.c_int32),
                ("max_new", ctypes.c_int32), ("max_len", ctypes.c_int32)]


class qp_paged_plan_info(ctypes.Structure):
    _fields_ = [("rows_per_tile", ctypes.c_int32), ("shares", ctypes.c_int32), ("key_chunks", ctypes.c_int32), ("chunk_entries", ctypes.c_int32),
                ("workgroups", ctypes.c_int32), ("scratch_bytes", ctypes.c_size_t)]


class qp_feed_stats(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("total_ms", ctypes.c_double), ("waited_ms", ctypes.c_double),
                ("first_group_wait_ms", ctypes.c_double)]


# qp_group_fn of include/qp_feed.h: (user, group, device_input, bytes, hip_stream) -> qp_status
GROUP_FN = ctypes.CFUNCTYPE(ctypes.c_int32, ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_size_t,
                            ctypes.c_void_p)
QP_FEED_PAGEABLE, QP_FEED_END, QP_FEED_TIMEOUT = 1, 100, 101


class qp_linear_plan_info(ctypes.Structure):
    _fields_ = [("token_rows_per_tile", ctypes.c_int32), ("workgroups", ctypes.c_int32), ("k_chunks", ctypes.c_int32),
                ("k_steps_per_chunk", ctypes.c_int32), ("scratch_bytes", ctypes.c_size_t)]


class QPError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status}, hip error {last_hip_error()})")


_lib = None
_vp, _i32, _i64, _f64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t
_LP, _CP = ctypes.POINTER(qp_layout), ctypes.POINTER(qp_cache)
_PC, _PB = ctypes.POINTER(qp_paged_cache), ctypes.POINTER(qp_paged_batch)
_SP, _WP, _f32 = ctypes.POINTER(qp_layer_shape), ctypes.POINTER(qp_layer_weights), ctypes.c_float

SIGNATURES = {
    "qp_keep_count": (_i64, [_i64, _f64]),
    "qp_cache_capacity": (_i64, [_i32, _i32, _i32, _f64]),
    "qp_debug_fail_after": (_i32, [_i32]),
    "qp_e4m3_from_bf16": (ctypes.c_uint8, [ctypes.c_uint16]),
    "qp_bf16_from_e4m3": (ctypes.c_uint16, [ctypes.c_uint8]),
    "qp_group_attend_noalloc": (_i32, [_LP, _vp, _vp, _vp, _i32, _CP, _vp, _vp, _vp]),
    "qp_group_bounds": (_i32, [_i32, _i32, _i32, ctypes.POINTER(_i32), ctypes.POINTER(_i32), _i32]),
    "qp_workspace_bytes": (_sz, [_LP, _i32, _i32]),
    "qp_group_attend": (_i32, [_LP, _vp, _vp, _vp, _i32, _CP, _vp, _vp, _vp, _sz, _vp]),
    "qp_score_kv": (_i32, [_LP, _i32, _vp, _vp, _i32, _vp, _i32, _vp, _vp, _sz, _vp]),
    "qp_topk_compact": (_i32, [_LP, _vp, _vp, _vp, _i32, _i32, _i32, _CP, _vp, _vp, _sz, _vp]),
    "qp_prefill_video": (_i32, [_LP, _i32, _i32, _i32, _f64, _i32, _vp, _vp, _vp, _vp, _i32, _CP, _vp, _vp, _sz, _vp]),
    "qp_attend_plan": (_i32, [_LP, _i32, _i32, _sz, ctypes.POINTER(qp_attend_plan_info)]),
    "qp_select_attend_kernel": (_i32, [_i32]),
    "qp_status_string": (ctypes.c_char_p, [_i32]),
    "qp_last_hip_error": (ctypes.c_int, []),
    "qp_version": (ctypes.c_char_p, []),
    # include/qp_layer.h
    "qp_rms_norm": (_i32, [_vp, _vp, _vp, _i32, _i32, _f32, _vp]),
    "qp_linear": (_i32, [_vp, _vp, _vp, _vp, _vp, _i32, _i32, _i32, _vp, _sz, _vp]),
    "qp_rope_table": (_i32, [_vp, _i64, _i32, _f32, ctypes.POINTER(ctypes.c_int32), _vp, _vp]),
    "qp_qkv_rope": (_i32, [_LP, _vp, _vp, _vp, _vp, _i32, _i32, _vp, _vp, _vp, _vp, _sz, _vp]),
    "qp_swiglu_gate_up": (_i32, [_vp, _vp, _vp, _i32, _i32, _i32, _vp]),
    "qp_select_linear_tile": (_i32, [_i32]),
    "qp_linear_plan": (_i32, [_i32, _i32, _i32, _sz, ctypes.POINTER(qp_linear_plan_info)]),
    "qp_layer_workspace_bytes": (_sz, [_LP, _SP, _i32, _i32]),
    "qp_layer_group": (_i32, [_LP, _SP, _WP, _vp, _vp, _i64, _i32, _i32, _vp, _i32, _i32, _i32, _CP, _vp, _vp, _vp,
                              _sz, _vp]),
    "qp_layer_window_queries": (_i32, [_LP, _SP, _WP, _vp, _vp, _i64, _i32, _vp, _vp, _sz, _vp]),
    # include/qp_paged.h
    "qp_paged_workspace_bytes": (_sz, [_LP, _i32, _i32, _i32, _i32, _i32]),
    "qp_paged_append": (_i32, [_LP, _PC, _PB, _vp, _vp, _i64, _i64, _vp, _i64, _i64, _i32, _vp]),
    "qp_paged_attend": (_i32, [_LP, _PC, _PB, _vp, _vp, _vp, _vp, _sz, _vp]),
    "qp_paged_weigh": (_i32, [_LP, _PC, _PB, _vp, _vp, _i32, _vp, _sz, _vp]),
    "qp_paged_evict": (_i32, [_LP, _PC, _PB, _i32, _i32, _i32, _vp, _i32, _vp, _vp, _vp, _sz, _vp]),
    "qp_paged_plan": (_i32, [_LP, _PC, _PB, _sz, ctypes.POINTER(qp_paged_plan_info)]),
    # include/qp_feed.h
    "qp_feed_create": (_i32, [_i32, _sz, _i32, ctypes.POINTER(_vp)]),
    "qp_feed_destroy": (None, [_vp]),
    "qp_feed_stop": (_i32, [_vp]),
    "qp_feed_begin_write": (_i32, [_vp, ctypes.POINTER(_vp)]),
    "qp_feed_publish": (_i32, [_vp, _sz]),
    "qp_feed_close": (_i32, [_vp]),
    "qp_feed_next": (_i32, [_vp, _i32, ctypes.POINTER(_vp), ctypes.POINTER(_sz), ctypes.POINTER(_i32)]),
    "qp_feed_release": (_i32, [_vp, _i32]),
    "qp_feed_consume": (_i32, [_vp, _vp, _vp, _sz, GROUP_FN, _vp, _vp, ctypes.POINTER(qp_feed_stats)]),
    "qp_feed_stub_producer": (_i32, [_vp, _vp, ctypes.POINTER(_sz), _i32, _i64, _i64]),
    "qp_feed_stub_join": (_i32, [_vp, ctypes.POINTER(_f64)]),
}


def lib():
    """The loaded C-ABI library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2505_16175_amd.build` "
                               "(or __graft_entry__.build()); there is no CPU fallback")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("expected a contiguous GPU tensor")
    return ctypes.c_void_p(t.data_ptr())


# The current stream's handle alone: torch.cuda.current_stream() builds a Stream object and looks its device up again, 3 of the
# 11 us that the host spends on a tiny video. Neither name is public: a torch without them takes the long way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream():
    if _raw_stream is None or _device is None:
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    return ctypes.c_void_p(_raw_stream(_device()))


def _check(status, where):
    if status != QP_OK:
        raise QPError(status, where)


def make_layout(n_q_heads, n_kv_heads, head_dim, dtype, softmax_scale=0.0) -> qp_layout:
    code = {torch.float32: QP_F32, torch.bfloat16: QP_BF16, "f32": QP_F32, "bf16": QP_BF16}[dtype]
    return qp_layout(n_q_heads, n_kv_heads, head_dim, code, softmax_scale)


class Cache:
    """Owner of the device buffers behind a qp_cache (torch allocates; the library only fills)."""

    def __init__(self, layout: qp_layout, capacity: int, device="cuda", fmt=QP_CACHE_SAME):
        """fmt = QP_CACHE_FP8_E4M3: K~ and V~ hold one E4M3 byte per element (torch.float8_e4m3fn is that format)."""
        dt = torch.float32 if layout.dtype == QP_F32 else torch.bfloat16
        if fmt == QP_CACHE_FP8_E4M3:
            dt = torch.float8_e4m3fn
        self.k = torch.zeros(layout.n_kv_heads, capacity, layout.head_dim, dtype=dt, device=device)
        self.v = torch.zeros_like(self.k)
        self.pos = torch.full((layout.n_kv_heads, capacity), -1, dtype=torch.int32, device=device)
        self.c = qp_cache(self.k.data_ptr(), self.v.data_ptr(), self.pos.data_ptr(), capacity, 0, fmt)

    @property
    def len(self):
        return self.c.len

    def reset(self):
        self.c.len = 0

    def nbytes(self):
        """Bytes of K and V actually held (2 * H_kv * len * d * sizeof)."""
        return 2 * self.k.shape[0] * self.c.len * self.k.shape[2] * self.k.element_size()


def status_string(status) -> str:
    return lib().qp_status_string(int(status)).decode()


def last_hip_error() -> int:
    return lib().qp_last_hip_error()


def version() -> str:
    return lib().qp_version().decode()


def keep_count(n_group_tokens, retention) -> int:
    return lib().qp_keep_count(n_group_tokens, retention)


def group_bounds(n_frames, tokens_per_frame, group_frames):
    """[(first_token, n_tokens)] of every frame-aligned group, from qp_group_bounds."""
    n = lib().qp_group_bounds(n_frames, tokens_per_frame, group_frames, None, None, 0)
    if n < 0:
        raise QPError(QP_ERR_INVALID_ARG, "qp_group_bounds")
    first, count = (ctypes.c_int32 * n)(), (ctypes.c_int32 * n)()
    lib().qp_group_bounds(n_frames, tokens_per_frame, group_frames, first, count, n)
    return [(int(f), int(c)) for f, c in zip(first, count)]


def cache_capacity(n_frames, tokens_per_frame, group_frames, retention) -> int:
    return lib().qp_cache_capacity(n_frames, tokens_per_frame, group_frames, retention)


def workspace_bytes(layout, max_group_tokens, n_window) -> int:
    return lib().qp_workspace_bytes(ctypes.byref(layout), max_group_tokens, n_window)


def make_workspace(layout, max_group_tokens, n_window, device="cuda") -> torch.Tensor:
    n = workspace_bytes(layout, max_group_tokens, n_window)
    if n == 0:
        raise QPError(QP_ERR_INVALID_ARG, "qp_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def attend_plan(layout, n_group_tokens, cache_len, workspace_bytes=0) -> dict:
    info = qp_attend_plan_info()
    _check(lib().qp_attend_plan(ctypes.byref(layout), n_group_tokens, cache_len, workspace_bytes, ctypes.byref(info)),
           "qp_attend_plan")
    return {name: getattr(info, name) for name, _ in qp_attend_plan_info._fields_}


def select_attend_kernel(which: int):
    _check(lib().qp_select_attend_kernel(which), "qp_select_attend_kernel")


def _ws(workspace):
    if workspace is None:
        return None, 0
    return _ptr(workspace), workspace.numel() * workspace.element_size()


def group_attend(layout, q_g, k_g, v_g, cache: Optional[Cache], out_g, lse=None, workspace=None):
    wp, wb = _ws(workspace)
    st = lib().qp_group_attend(ctypes.byref(layout), _ptr(q_g), _ptr(k_g), _ptr(v_g), q_g.shape[0],
                               ctypes.byref(cache.c) if cache is not None else None, _ptr(out_g), _ptr(lse),
                               wp, wb, _stream())
    _check(st, "qp_group_attend")


NOALLOC_SCRATCH_BYTES = 8 << 20
NOALLOC_MAX_ROWS = 2048


def group_attend_noalloc(layout, q_g, k_g, v_g, cache: Optional[Cache], out_g, lse=None):
    st = lib().qp_group_attend_noalloc(ctypes.byref(layout), _ptr(q_g), _ptr(k_g), _ptr(v_g), q_g.shape[0],
                                       ctypes.byref(cache.c) if cache is not None else None, _ptr(out_g), _ptr(lse),
                                       _stream())
    _check(st, "qp_group_attend_noalloc")


def score_kv(layout, rule, k_g, v_g, q_win, scores, workspace=None):
    wp, wb = _ws(workspace)
    n_g = (k_g if k_g is not None else v_g).shape[0]
    st = lib().qp_score_kv(ctypes.byref(layout), RULES.get(rule, rule), _ptr(k_g), _ptr(v_g), n_g, _ptr(q_win),
                           0 if q_win is None else q_win.shape[0], _ptr(scores), wp, wb, _stream())
    _check(st, "qp_score_kv")


def topk_compact(layout, scores, k_g, v_g, keep, group_token_base, cache: Cache, kept_idx=None, workspace=None):
    wp, wb = _ws(workspace)
    st = lib().qp_topk_compact(ctypes.byref(layout), _ptr(scores), _ptr(k_g), _ptr(v_g), k_g.shape[0], keep,
                               group_token_base, ctypes.byref(cache.c), _ptr(kept_idx), wp, wb, _stream())
    _check(st, "qp_topk_compact")


def prefill_video(layout, n_frames, tokens_per_frame, group_frames, retention, rule, q, k, v, q_win, cache: Cache,
                  out, workspace):
    wp, wb = _ws(workspace)
    st = lib().qp_prefill_video(ctypes.byref(layout), n_frames, tokens_per_frame, group_frames, retention,
                                RULES.get(rule, rule), _ptr(q), _ptr(k), _ptr(v), _ptr(q_win),
                                0 if q_win is None else q_win.shape[0], ctypes.byref(cache.c), _ptr(out), wp, wb,
                                _stream())
    _check(st, "qp_prefill_video")


# ---- include/qp_layer.h: the decoder layer around the path -------------------------------------------------
def make_layer_shape(d_model, d_ff, rms_eps=1e-6, rope_theta=1e6, mrope_section=(16, 24, 24)) -> qp_layer_shape:
    return qp_layer_shape(d_model, d_ff, rms_eps, rope_theta, (ctypes.c_int32 * 3)(*mrope_section))


class LayerWeights:
    """Keeps a layer's weight tensors alive next to the qp_layer_weights struct that points at them."""

    def __init__(self, ln1_w, w_qkv, b_qkv, w_o, ln2_w, w_gate_up, w_down):
        self.tensors = dict(ln1_w=ln1_w, w_qkv=w_qkv, b_qkv=b_qkv, w_o=w_o, ln2_w=ln2_w, w_gate_up=w_gate_up,
                            w_down=w_down)
        self.c = qp_layer_weights(**{name: _ptr(t).value for name, t in self.tensors.items()})


def rms_norm(x, w, out, eps):
    _check(lib().qp_rms_norm(_ptr(x), _ptr(w), _ptr(out), x.shape[0], x.shape[1], eps, _stream()), "qp_rms_norm")


def linear(x, w, bias, residual, out, workspace=None):
    wp, wb = _ws(workspace)
    _check(lib().qp_linear(_ptr(x), _ptr(w), _ptr(bias), _ptr(residual), _ptr(out), x.shape[0], w.shape[0], x.shape[1],
                           wp, wb, _stream()), "qp_linear")


def _pos_ptr(pos, first, axis_stride):
    """pos: int32 [3][N] on the GPU; the group starts at token `first`."""
    if pos.dtype != torch.int32 or not pos.is_cuda or not pos.is_contiguous() or pos.shape[0] != 3:
        raise ValueError("expected a contiguous int32 [3][N] GPU tensor of position indices")
    return ctypes.c_void_p(pos.data_ptr() + 4 * first), (pos.shape[1] if axis_stride is None else axis_stride)


def rope_table(pos, first, n_tokens, theta, mrope_section, cos_sin):
    pp, stride = _pos_ptr(pos, first, None)
    _check(lib().qp_rope_table(pp, stride, n_tokens, theta, (ctypes.c_int32 * 3)(*mrope_section), _ptr(cos_sin),
                               _stream()), "qp_rope_table")


def qkv_rope(layout, h, w_qkv, b_qkv, cos_sin, q, k, v, workspace=None):
    wp, wb = _ws(workspace)
    _check(lib().qp_qkv_rope(ctypes.byref(layout), _ptr(h), _ptr(w_qkv), _ptr(b_qkv), _ptr(cos_sin), h.shape[0],
                             h.shape[1], _ptr(q), _ptr(k), _ptr(v), wp, wb, _stream()), "qp_qkv_rope")


def swiglu_gate_up(h, w_gate_up, act):
    _check(lib().qp_swiglu_gate_up(_ptr(h), _ptr(w_gate_up), _ptr(act), h.shape[0], h.shape[1],
                                   w_gate_up.shape[0] // 2, _stream()), "qp_swiglu_gate_up")


def linear_plan(m, n, k, workspace_bytes=0) -> dict:
    info = qp_linear_plan_info()
    _check(lib().qp_linear_plan(m, n, k, workspace_bytes, ctypes.byref(info)), "qp_linear_plan")
    return {name: getattr(info, name) for name, _ in qp_linear_plan_info._fields_}


def select_linear_tile(token_rows: int):
    _check(lib().qp_select_linear_tile(token_rows), "qp_select_linear_tile")


def layer_workspace_bytes(layout, shape, max_group_tokens, n_window) -> int:
    return lib().qp_layer_workspace_bytes(ctypes.byref(layout), ctypes.byref(shape), max_group_tokens, n_window)


def make_layer_workspace(layout, shape, max_group_tokens, n_window, device="cuda") -> torch.Tensor:
    n = layer_workspace_bytes(layout, shape, max_group_tokens, n_window)
    if n == 0:
        raise QPError(QP_ERR_INVALID_ARG, "qp_layer_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def layer_group(layout, shape, weights: LayerWeights, x_g, pos, first, group_token_base, q_win, rule, keep,
                cache: Cache, x_out, kept_idx, workspace):
    wp, wb = _ws(workspace)
    pp, stride = _pos_ptr(pos, first, None)
    st = lib().qp_layer_group(ctypes.byref(layout), ctypes.byref(shape), ctypes.byref(weights.c), _ptr(x_g), pp, stride,
                              x_g.shape[0], group_token_base, _ptr(q_win), 0 if q_win is None else q_win.shape[0],
                              RULES.get(rule, rule), keep, ctypes.byref(cache.c), _ptr(x_out), _ptr(kept_idx), wp, wb,
                              _stream())
    _check(st, "qp_layer_group")


def layer_window_queries(layout, shape, weights: LayerWeights, x_win, pos_win, q_win_out, workspace):
    wp, wb = _ws(workspace)
    pp, stride = _pos_ptr(pos_win, 0, None)
    st = lib().qp_layer_window_queries(ctypes.byref(layout), ctypes.byref(shape), ctypes.byref(weights.c), _ptr(x_win),
                                       pp, stride, x_win.shape[0], _ptr(q_win_out), wp, wb, _stream())
    _check(st, "qp_layer_window_queries")


# ---- include/qp_feed.h: the consumer side of the loader / prefill pipeline ----------------------------------
class Feed:
    """Owner of a qp_feed handle. Producer calls may come from any Python thread (ctypes drops the GIL while a
    call blocks); consume() runs the consumer loop on the calling thread."""

    def __init__(self, n_slots, slot_bytes, flags=0):
        self.h = ctypes.c_void_p()
        _check(lib().qp_feed_create(n_slots, slot_bytes, flags, ctypes.byref(self.h)), "qp_feed_create")
        self.slot_bytes = slot_bytes
        self._keep = []

    def destroy(self):
        if self.h:
            lib().qp_feed_destroy(self.h)
            self.h = ctypes.c_void_p()

    def begin_write(self) -> int:
        p = ctypes.c_void_p()
        _check(lib().qp_feed_begin_write(self.h, ctypes.byref(p)), "qp_feed_begin_write")
        return p.value

    def publish(self, nbytes):
        _check(lib().qp_feed_publish(self.h, nbytes), "qp_feed_publish")

    def close(self):
        _check(lib().qp_feed_close(self.h), "qp_feed_close")

    def stop(self):
        _check(lib().qp_feed_stop(self.h), "qp_feed_stop")

    def next(self, timeout_ms=-1):
        """(status, host_pointer, bytes, group); status is QP_OK, QP_FEED_END or QP_FEED_TIMEOUT."""
        p, n, g = ctypes.c_void_p(), ctypes.c_size_t(), ctypes.c_int32()
        st = lib().qp_feed_next(self.h, timeout_ms, ctypes.byref(p), ctypes.byref(n), ctypes.byref(g))
        if st not in (QP_OK, QP_FEED_END, QP_FEED_TIMEOUT):
            raise QPError(st, "qp_feed_next")
        return st, p.value, n.value, g.value

    def release(self, group):
        _check(lib().qp_feed_release(self.h, group), "qp_feed_release")

    def consume(self, buf0, buf1, group_fn) -> dict:
        """group_fn(group, device_pointer, nbytes) enqueues the group's work on torch's current stream."""
        failure = []

        def tramp(_user, group, dev, nbytes, _stream):
            # an exception cannot cross the C frames of qp_feed_consume: stop the run and re-raise it afterwards
            try:
                group_fn(group, dev, nbytes)
                return QP_OK
            except QPError as e:
                failure.append(e)
                return e.status
            except BaseException as e:  # noqa: BLE001
                failure.append(e)
                return QP_ERR_INVALID_ARG
        cb = GROUP_FN(tramp)
        stats = qp_feed_stats()
        st = lib().qp_feed_consume(self.h, _ptr(buf0), _ptr(buf1), buf0.numel() * buf0.element_size(), cb, None,
                                   _stream(), ctypes.byref(stats))
        if failure:
            raise failure[0]
        _check(st, "qp_feed_consume")
        return {name: getattr(stats, name) for name, _ in qp_feed_stats._fields_}

    def stub_producer(self, host_src: torch.Tensor, bytes_per_group, first_latency_us, per_group_latency_us):
        """host_src: contiguous CPU tensor holding the groups back to back."""
        arr = (ctypes.c_size_t * len(bytes_per_group))(*bytes_per_group)
        self._keep = [host_src, arr]
        _check(lib().qp_feed_stub_producer(self.h, ctypes.c_void_p(host_src.data_ptr()), arr, len(bytes_per_group),
                                           first_latency_us, per_group_latency_us), "qp_feed_stub_producer")

    def stub_join(self) -> float:
        ms = ctypes.c_double()
        _check(lib().qp_feed_stub_join(self.h, ctypes.byref(ms)), "qp_feed_stub_join")
        return ms.value


# ---- the paged cache (include/qp_paged.h) ----
# A decoding step's calls are a few microseconds of GPU work, so what the host spends on one counts: what does not change from call to
# call (the structs' references) is kept with its owner, and a tensor is looked at once.

def _here():
    return torch.cuda.current_device() if _device is None else _device()


def _dense(t, dtype, shape, name, here):
    """The address of a dense tensor of that type and shape on the current device (one of another device would be read across the
    link, or not at all)."""
    if t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{name}: expected {dtype} {tuple(shape)}, got {t.dtype} {tuple(t.shape)}")
    if t.get_device() != here or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous tensor of the current GPU")
    return t.data_ptr()


def _scratch(workspace, here):
    if workspace is None:
        return None, 0
    if workspace.get_device() != here or not workspace.is_contiguous():
        raise ValueError("workspace: expected a contiguous tensor of the current GPU")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _layout_dtype(layout):
    return torch.float32 if layout.dtype == QP_F32 else torch.bfloat16


class PagedCache:
    """Owner of the device buffers behind a qp_paged_cache: a pool of pages that many sequences share."""

    def __init__(self, layout: qp_layout, n_pages: int, page_tokens: int, device="cuda", fmt=QP_CACHE_SAME, weights=True,
                 k=None, v=None, pos=None, weight=None):
        """New zeroed buffers (positions -1), or the caller's own: k, v [n_pages][H_kv][page_tokens][d] in the layout's dtype
        or torch.float8_e4m3fn, pos int32 and weight float32 [n_pages][H_kv][page_tokens]. weights=False: a pool without them,
        which paged_weigh and paged_evict refuse."""
        rows = (n_pages, layout.n_kv_heads, page_tokens)
        if k is not None and k.dtype == torch.float8_e4m3fn:
            fmt = QP_CACHE_FP8_E4M3
        dt = torch.float8_e4m3fn if fmt == QP_CACHE_FP8_E4M3 else _layout_dtype(layout)
        self.k = torch.zeros(*rows, layout.head_dim, dtype=dt, device=device) if k is None else k
        self.v = torch.zeros(*rows, layout.head_dim, dtype=dt, device=device) if v is None else v
        self.pos = torch.full(rows, -1, dtype=torch.int32, device=device) if pos is None else pos
        self.weight = torch.zeros(rows, dtype=torch.float32, device=device) if weights and weight is None else weight
        here = self.k.get_device()
        at = [_dense(t, d, (*rows, layout.head_dim) if t is self.k or t is self.v else rows, name, here)
              for t, d, name in ((self.k, dt, "k"), (self.v, dt, "v"), (self.pos, torch.int32, "pos"))]
        at.append(None if self.weight is None else _dense(self.weight, torch.float32, rows, "weight", here))
        self.device_index = here
        self.made_for = (layout.n_kv_heads, layout.head_dim, layout.dtype)
        self.c = qp_paged_cache(*at, n_pages, page_tokens, fmt)
        self.ref = ctypes.byref(self.c)


class PagedBatch:
    """The sequences of a call: page_table int32 [n_seqs][pages], length int32 [n_seqs] and row_start int32 [n_seqs + 1] on the
    GPU (their values may change between calls, and between replays of a captured one). max_new and max_len bound what is
    launched; by default every row may belong to one sequence, and a sequence may fill its table."""

    def __init__(self, page_table, length, row_start=None, n_rows=0, max_new=None, max_len=None):
        here = page_table.get_device()
        if page_table.dim() != 2:
            raise ValueError("page_table: expected int32 [n_seqs][pages]")
        n_seqs = page_table.shape[0]
        at = [_dense(page_table, torch.int32, page_table.shape, "page_table", here),
              _dense(length, torch.int32, (n_seqs,), "length", here),
              None if row_start is None else _dense(row_start, torch.int32, (n_seqs + 1,), "row_start", here)]
        if here < 0:
            raise ValueError("page_table: expected a tensor on the GPU")
        self.page_table, self.length, self.row_start, self.max_len = page_table, length, row_start, max_len
        self.n_seqs, self.n_rows, self.device_index = n_seqs, n_rows, here
        self.c = qp_paged_batch(*at, n_seqs, page_table.shape[1], n_rows, n_rows if max_new is None else max_new, max_len or 0)
        self.ref = ctypes.byref(self.c)
        self.refs = {}                                   # page_tokens -> a struct of its own, where no max_len is stated

    def of(self, cache):
        """The struct for a pool, whose pages say what a sequence of the batch can hold where it states no max_len. A struct once
        handed out is never written again: calls run without the interpreter's lock, and another thread's may be reading it."""
        if self.max_len is not None:
            return self.ref
        page_tokens = cache.c.page_tokens
        ref = self.refs.get(page_tokens)
        if ref is None:
            c = qp_paged_batch.from_buffer_copy(self.c)
            c.max_len = min(c.table_pages * page_tokens, 1 << 30)
            ref = self.refs[page_tokens] = ctypes.byref(c)
        return ref


def _same_gpu(layout, cache, batch):
    if cache.made_for != (layout.n_kv_heads, layout.head_dim, layout.dtype):
        raise ValueError("expected a cache of this layout's heads and dtype")
    here = _here()
    if cache.device_index != here or batch.device_index != here:
        raise ValueError("expected a cache and a batch of the current GPU")
    return here


def paged_workspace_bytes(layout, n_seqs, n_rows, max_new, max_len, keep=0) -> int:
    return lib().qp_paged_workspace_bytes(ctypes.byref(layout), n_seqs, n_rows, max_new, max_len, keep)


def make_paged_workspace(layout, batch: PagedBatch, keep=0, page_tokens=256, device="cuda") -> torch.Tensor:
    """Scratch for every paged call of the batch's sizes (page_tokens: needed where the batch states no max_len)."""
    max_len = min(batch.c.table_pages * page_tokens, 1 << 30) if batch.max_len is None else batch.max_len
    n = paged_workspace_bytes(layout, batch.n_seqs, batch.n_rows, batch.c.max_new, max_len, keep)
    if n == 0:
        raise QPError(QP_ERR_INVALID_ARG, "qp_paged_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=device)


def paged_append(layout, cache: PagedCache, batch: PagedBatch, k, v, pos):
    """k, v [n_rows][H_kv][d] of any strides whose rows are runs of d elements (a flat cache's [H_kv][capacity][d] comes as
    k.transpose(0, 1)[:n]); pos int32 [n_rows], or [n_rows][H_kv] with a position per head. Rows of an 8-bit pool may be
    torch.float8_e4m3fn already."""
    here = _same_gpu(layout, cache, batch)
    n, h_kv, d = batch.n_rows, layout.n_kv_heads, layout.head_dim
    shape, dt = (n, h_kv, d), k.dtype
    raw = dt is torch.float8_e4m3fn
    if not raw and dt is not _layout_dtype(layout) or v.dtype is not dt or k.shape != shape or v.shape != shape:
        raise ValueError(f"k and v: expected {_layout_dtype(layout)} {shape}, got {dt} {tuple(k.shape)} and {v.dtype} {tuple(v.shape)}")
    sk, sv = k.stride(), v.stride()
    if n == 1 or h_kv == 1:                              # of one row, any stride does
        sk, sv = ((0 if n == 1 else s[0], 0 if h_kv == 1 else s[1], s[2]) for s in (sk, sv))
    if sk != sv or sk[2] != 1:
        raise ValueError("k and v: expected the same strides and rows in one run")
    if pos.dtype is not torch.int32 or pos.shape != shape[:1] and pos.shape != shape[:2]:
        raise ValueError("pos: expected int32 [n_rows] or [n_rows][H_kv]")
    if k.get_device() != here or v.get_device() != here or pos.get_device() != here:
        raise ValueError("expected tensors of the current GPU")
    sp = pos.stride()
    st = lib().qp_paged_append(ctypes.byref(layout), cache.ref, batch.of(cache), k.data_ptr(), v.data_ptr(), sk[0], sk[1],
                               pos.data_ptr(), sp[0], sp[1] if len(sp) == 2 else 0, QP_CACHE_FP8_E4M3 if raw else QP_CACHE_SAME,
                               _stream())
    _check(st, "qp_paged_append")


def paged_attend(layout, cache: PagedCache, batch: PagedBatch, q, out, lse=None, workspace=None):
    """q, out [n_rows][H_q][d], lse float32 [H_q][n_rows]."""
    here = _same_gpu(layout, cache, batch)
    dt, shape = _layout_dtype(layout), (batch.n_rows, layout.n_q_heads, layout.head_dim)
    wp, wb = _scratch(workspace, here)
    st = lib().qp_paged_attend(ctypes.byref(layout), cache.ref, batch.of(cache), _dense(q, dt, shape, "q", here),
                               _dense(out, dt, shape, "out", here),
                               None if lse is None else _dense(lse, torch.float32, (shape[1], shape[0]), "lse", here), wp, wb, _stream())
    _check(st, "qp_paged_attend")


def paged_weigh(layout, cache: PagedCache, batch: PagedBatch, q, lse, accumulate=True, workspace=None):
    """Adds to (or, accumulate=False, writes) cache.weight what the batch's rows of paged_attend's lse looked at."""
    here = _same_gpu(layout, cache, batch)
    shape = (batch.n_rows, layout.n_q_heads, layout.head_dim)
    wp, wb = _scratch(workspace, here)
    st = lib().qp_paged_weigh(ctypes.byref(layout), cache.ref, batch.of(cache), _dense(q, _layout_dtype(layout), shape, "q", here),
                              _dense(lse, torch.float32, (shape[1], shape[0]), "lse", here), 1 if accumulate else 0, wp, wb, _stream())
    _check(st, "qp_paged_weigh")


def paged_evict(layout, cache: PagedCache, batch: PagedBatch, keep, n_first, n_last, to_table, to_len, kept=None, workspace=None):
    """to_table int32 [n_seqs][pages], to_len int32 [n_seqs], kept int32 [n_seqs][H_kv][keep] or None."""
    here = _same_gpu(layout, cache, batch)
    n_seqs = batch.n_seqs
    if to_table.dim() != 2 or to_table.shape[0] != n_seqs:
        raise ValueError("to_table: expected int32 [n_seqs][pages]")
    wp, wb = _scratch(workspace, here)
    st = lib().qp_paged_evict(ctypes.byref(layout), cache.ref, batch.of(cache), keep, n_first, n_last,
                              _dense(to_table, torch.int32, to_table.shape, "to_table", here), to_table.shape[1],
                              _dense(to_len, torch.int32, (n_seqs,), "to_len", here),
                              None if kept is None else _dense(kept, torch.int32, (n_seqs, layout.n_kv_heads, keep), "kept", here),
                              wp, wb, _stream())
    _check(st, "qp_paged_evict")


def paged_plan(layout, cache: PagedCache, batch: PagedBatch, workspace_bytes=0) -> dict:
    info = qp_paged_plan_info()
    _check(lib().qp_paged_plan(ctypes.byref(layout), cache.ref, batch.of(cache), workspace_bytes, ctypes.byref(info)), "qp_paged_plan")
    return {name: getattr(info, name) for name, _ in qp_paged_plan_info._fields_}
