"""ctypes binding of libpad (include/pad.h): argument marshalling only.

Every step of the decode path runs in the CUDA library; this module converts
torch tensors to device pointers, numpy arrays to host pointers, and status
codes to exceptions.  It fails loudly when libpad.so has not been built.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_float, c_int32, c_int64, c_size_t, c_uint8, c_void_p

import numpy as np

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpad.so")
_lib = None

PAD_OK = 0
STATUS_NAMES = {
    0: "PAD_OK", 1: "PAD_ERR_INVALID_ARG", 2: "PAD_ERR_UNSUPPORTED", 3: "PAD_ERR_OUT_OF_PAGES",
    4: "PAD_ERR_WORKSPACE_TOO_SMALL", 5: "PAD_ERR_CUDA", 6: "PAD_ERR_DEVICE_TIMEOUT",
    7: "PAD_ERR_DEVICE_BOUNDS",
}
FLAG_PREFIX_SIMT = 0x1
FLAG_PREFIX_MMA = 0x2
FLAG_PREFIX_TC = 0x4
FLAG_FUSED_MERGE = 0x8
FLAG_PREFIX_DUAL = 0x10
G_ALL = 0
G_SELF = 1
BRANCH_OWN = 0
BRANCH_CAUSAL = 1
KV_BF16 = 0
KV_FP8 = 1
KV_FP4 = 4


class PadError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


class Problem(ctypes.Structure):
    _fields_ = [("h_q", c_int32), ("h_kv", c_int32), ("head_dim", c_int32),
                ("page_size", c_int32), ("scale", c_float), ("out_dtype", c_int32),
                ("num_sms", c_int32), ("flags", c_int32)]


class PlanInfo(ctypes.Structure):
    _fields_ = [("n_videos", c_int32), ("n_events", c_int32), ("n_work_items", c_int32),
                ("split_len", c_int32), ("prefix_kernel", c_int32), ("n_new_pages", c_int32),
                ("partial_rows", c_int64), ("workspace_bytes", c_int64),
                ("param_descriptor_bytes", c_int32), ("fused_tail", c_int32),
                ("generation", ctypes.c_uint64), ("prefix_ctas", c_int32), ("max_split_tiles", c_int32),
                ("merge_first", c_int32)]


class ChunkInfo(ctypes.Structure):
    _fields_ = [("n_tokens", c_int64), ("n_cached", c_int64), ("n_drafts", c_int64), ("workspace_bytes", c_int64),
                ("partial_rows", c_int64), ("n_new_pages", c_int32), ("prefix_splits", c_int32),
                ("page_splits", c_int32), ("tc_items", c_int32), ("mma_items", c_int32), ("prefix_tokens", c_int32)]


class RopeSpec(ctypes.Structure):
    _fields_ = [("head_dim", c_int32), ("rotary_dim", c_int32), ("layout", c_int32), ("scaling", c_int32)] + [
        (f, ctypes.c_double) for f in ("theta", "factor", "original_len", "low", "high", "magnitude")]


class RopeTurns(ctypes.Structure):
    _fields_ = [("head_dim", c_int32), ("rotary_dim", c_int32), ("layout", c_int32), ("magnitude", c_float),
                ("turn", ctypes.c_uint64 * 64)]


_I32P = POINTER(c_int32)
_I64P = POINTER(c_int64)

# name -> (restype, argtypes); mirrors include/pad.h
_SIGNATURES = {
    "pad_cache_state_create": (c_int32, [c_int32, POINTER(c_void_p)]),
    "pad_cache_state_destroy": (None, [c_void_p]),
    "pad_cache_state_mark_used": (c_int32, [c_void_p, _I32P, c_int32]),
    "pad_cache_state_release": (c_int32, [c_void_p, _I32P, c_int32]),
    "pad_cache_state_num_pages": (c_int32, [c_void_p]),
    "pad_cache_state_free_count": (c_int32, [c_void_p]),
    "pad_cache_state_export": (c_int32, [c_void_p, POINTER(c_uint8)]),
    "pad_cache_state_import": (c_int32, [c_void_p, POINTER(c_uint8), c_int32]),
    "pad_workspace_size": (c_size_t, [POINTER(Problem), c_int32, _I32P, c_int32, _I32P]),
    "pad_plan": (c_int32, [POINTER(Problem), c_void_p, c_int32, _I32P, _I64P, c_int32, _I32P,
                           _I32P, c_void_p, c_int32, c_void_p, c_size_t, c_void_p,
                           POINTER(c_void_p)]),
    "pad_plan_new_pages": (c_int32, [c_void_p, _I32P]),
    "pad_plan_release_new_pages": (c_int32, [c_void_p, c_void_p]),
    "pad_step_create": (c_int32, [POINTER(Problem), c_void_p, c_int32, _I32P, _I64P, c_int32, _I32P, _I32P,
                                  c_void_p, c_int32, c_void_p, c_size_t] + [c_void_p] * 10
                        + [c_int32, POINTER(c_void_p)]),
    "pad_step_set_rope": (c_int32, [c_void_p, _I32P, c_void_p, c_int32]),
    "pad_step_set_g_visibility": (c_int32, [c_void_p, c_int32, _I32P, _I32P]),
    "pad_step_set_branch_visibility": (c_int32, [c_void_p, c_int32]),
    "pad_step_run": (c_int32, [c_void_p, _I32P]),
    "pad_step_run_host": (c_int32, [c_void_p] * 6 + [_I32P]),
    "pad_step_destroy": (None, [c_void_p]),
    "pad_plan_set_rope": (c_int32, [c_void_p, _I32P, c_void_p, c_int32]),
    "pad_plan_set_g_visibility": (c_int32, [c_void_p, c_int32, _I32P, _I32P]),
    "pad_plan_set_branch_visibility": (c_int32, [c_void_p, c_int32]),
    "pad_plan_get_info": (c_int32, [c_void_p, POINTER(PlanInfo)]),
    "pad_plan_destroy": (c_int32, [c_void_p]),
    "pad_kv_append": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "pad_event_decode_attn": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                        c_void_p, c_void_p, c_void_p, c_void_p]),
    "pad_event_decode_attn_static": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                               c_void_p, c_void_p, c_void_p, c_void_p]),
    "pad_decode_step": (c_int32, [c_void_p] * 11),
    "pad_prefill_attn": (c_int32, [POINTER(Problem), c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p, c_void_p, c_void_p]),
    "pad_prefill_status": (c_int32, [c_void_p]),
    "pad_ground_pool": (c_int32, [c_void_p, c_int64, c_int32, c_void_p, c_int32, c_void_p, c_void_p]),
    "pad_ground_score": (c_int32, [c_void_p, c_int32, c_void_p, c_int32, c_int32, c_float, c_void_p, c_void_p,
                                   c_void_p, c_void_p]),
    "pad_attn_aggregate": (c_int32, [c_void_p, c_int64, c_int32, c_void_p, c_void_p, c_int32, c_void_p, c_int32,
                                     c_void_p, c_void_p, ctypes.c_size_t, c_void_p, c_void_p]),
    "pad_attn_aggregate_workspace_size": (ctypes.c_size_t, [c_int64, c_int32, c_int32]),
    "pad_chunk_workspace_size": (c_size_t, [POINTER(Problem), c_int32, c_int32, _I32P, c_int32, _I32P, _I32P, _I32P]),
    "pad_chunk_plan": (c_int32, [POINTER(Problem), c_int32, c_void_p, c_int32, _I32P, _I64P, c_int32, _I32P, _I32P, _I32P,
                                 c_void_p, c_int32, c_int32, c_void_p, c_size_t, c_void_p, POINTER(c_void_p)]),
    "pad_chunk_get_info": (c_int32, [c_void_p, POINTER(ChunkInfo)]),
    "pad_chunk_new_pages": (c_int32, [c_void_p, _I32P, _I32P, _I32P]),
    "pad_chunk_destroy": (c_int32, [c_void_p]),
    "pad_chunk_append": (c_int32, [c_void_p, c_void_p, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_void_p]),
    "pad_rope_init": (c_int32, [POINTER(RopeSpec), POINTER(RopeTurns)]),
    "pad_chunk_append_rope": (c_int32, [c_void_p, POINTER(RopeTurns), c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p,
                                        c_void_p, c_int64] + [c_void_p] * 5),
    "pad_chunk_probs": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                  c_void_p, c_void_p, c_int32, c_void_p, c_void_p, c_int64, c_int32, c_void_p, c_int64, c_void_p]),
    "pad_chunk_read": (c_int32, [c_void_p] * 8),
    "pad_chunk_attn": (c_int32, [c_void_p, c_void_p, c_int64] + [c_void_p] * 9),
    "pad_draft_verify": (c_int32, [c_void_p, c_int32, c_int32, c_void_p, c_int64, c_void_p, c_int64] + [c_void_p] * 6),
    "pad_chunk_commit": (c_int32, [c_void_p, c_void_p, _I32P, _I32P]),
    "pad_chunk_status": (c_int32, [c_void_p, c_void_p]),
    "pad_device_status": (c_int32, [c_void_p, c_void_p]),
    "pad_last_error": (ctypes.c_char_p, []),
    "pad_status_string": (ctypes.c_char_p, [c_int32]),
    "pad_step_enqueue_host": (c_int32, [c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p, _I32P]),
    "pad_step_wait": (c_int32, [c_void_p]),
    "pad_step_profile": (c_int32, [c_void_p, c_int32]),
    "pad_step_profile_read": (c_int32, [c_void_p, POINTER(ctypes.c_double), c_int32]),
    "pad_timing_enable": (c_int32, [c_int32]),
    "pad_timing_read": (c_int32, [POINTER(c_float), _I32P]),
}


def lib_path() -> str:
    return _LIB_PATH


def lib():
    """Load libpad.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"libpad.so is not built ({_LIB_PATH}); run "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        L = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def _check(status: int):
    if status != PAD_OK:
        msg = lib().pad_last_error().decode(errors="replace")
        raise PadError(status, msg)


def _i32(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(_I32P)


def _host(a, dtype):
    """A contiguous host array and its address (a fraction of ctypes.data_as's cost)."""
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.__array_interface__["data"][0]


def _ptr(t):
    """Device pointer of a tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors passed to libpad must be contiguous")
    return c_void_p(t.data_ptr())


_raw_stream = None


def _current_stream() -> int:
    """Handle of the current device's current stream.  torch.cuda.current_stream() builds a
    Stream object for it (3 us per call); the raw handle takes 0.2 us where torch offers it."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        dev = getattr(torch._C, "_cuda_getDevice", None)
        if get is not None and dev is not None:
            _raw_stream = lambda: get(dev())
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream
    return _raw_stream()


def _stream(stream):
    if stream is None:
        return c_void_p(_current_stream())
    if isinstance(stream, int):
        return c_void_p(stream)
    return c_void_p(stream.cuda_stream)


def _stream_handle(stream):
    """The handle that _stream wraps, as an integer."""
    if stream is None:
        return _raw_stream() if _raw_stream is not None else _current_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def make_problem(h_q, h_kv, head_dim, page_size=16, scale=None, out_dtype=0, num_sms=0, flags=0):
    if scale is None:
        scale = 1.0 / float(head_dim) ** 0.5
    return Problem(h_q, h_kv, head_dim, page_size, scale, out_dtype, num_sms, flags)


class CacheState:
    """Host bookkeeping of the private-KV page pool (pad_cache_state)."""

    def __init__(self, n_pages: int, used_pages=None):
        h = c_void_p()
        _check(lib().pad_cache_state_create(int(n_pages), ctypes.byref(h)))
        self._h = h
        if used_pages is not None and len(used_pages):
            self.mark_used(used_pages)

    @property
    def handle(self):
        return self._h

    def mark_used(self, pages):
        a, p = _i32(pages)
        _check(lib().pad_cache_state_mark_used(self._h, p, int(a.size)))

    def release(self, pages):
        a, p = _i32(pages)
        _check(lib().pad_cache_state_release(self._h, p, int(a.size)))

    @property
    def n_pages(self) -> int:
        return int(lib().pad_cache_state_num_pages(self._h))

    @property
    def free_count(self) -> int:
        return int(lib().pad_cache_state_free_count(self._h))

    def export(self) -> np.ndarray:
        out = np.zeros(self.n_pages, dtype=np.uint8)
        _check(lib().pad_cache_state_export(self._h, out.ctypes.data_as(POINTER(c_uint8))))
        return out

    def import_(self, used: np.ndarray):
        u = np.ascontiguousarray(used, dtype=np.uint8)
        _check(lib().pad_cache_state_import(self._h, u.ctypes.data_as(POINTER(c_uint8)), int(u.size)))

    def free_pages(self) -> np.ndarray:
        return np.nonzero(self.export() == 0)[0].astype(np.int32)

    def __del__(self):
        if getattr(self, "_h", None) is not None and _lib is not None:
            _lib.pad_cache_state_destroy(self._h)
            self._h = None


class Plan:
    """A planned decode step (pad_plan_t)."""

    def __init__(self, handle, n_events):
        self._h = handle
        self.n_events = n_events

    @property
    def handle(self):
        return self._h

    def new_pages(self) -> np.ndarray:
        out = np.full(self.n_events, -1, dtype=np.int32)
        _check(lib().pad_plan_new_pages(self._h, out.ctypes.data_as(_I32P)))
        return out

    def release_new_pages(self, cache: "CacheState"):
        """Give the pages this plan took back to ``cache`` (pad_plan_release_new_pages)."""
        _check(lib().pad_plan_release_new_pages(self._h, cache.handle))

    def set_rope(self, positions, cos_sin, max_position: int = None):
        """Rotate q and k_new at these per-event positions in the step's kernels
        (pad_plan_set_rope); ``cos_sin`` is the device fp32 table [max_position, D]."""
        pos = np.ascontiguousarray(positions, dtype=np.int32)
        n = int(cos_sin.shape[0]) if max_position is None else int(max_position)
        _check(lib().pad_plan_set_rope(self._h, pos.ctypes.data_as(_I32P), _ptr(cos_sin), n))

    def set_g_visibility(self, mode: int, n_planning=None, g_index=None):
        """pad_plan_set_g_visibility: G_SELF hides the other events' planning tokens."""
        if n_planning is None or g_index is None:
            _check(lib().pad_plan_set_g_visibility(self._h, int(mode), None, None))
            return
        k = np.ascontiguousarray(n_planning, dtype=np.int32)
        g = np.ascontiguousarray(g_index, dtype=np.int32)
        _check(lib().pad_plan_set_g_visibility(self._h, mode, k.ctypes.data_as(_I32P),
                                               g.ctypes.data_as(_I32P)))

    def set_branch_visibility(self, mode: int):
        """pad_plan_set_branch_visibility: BRANCH_CAUSAL shows every branch's stored tokens."""
        _check(lib().pad_plan_set_branch_visibility(self._h, int(mode)))

    def info(self) -> dict:
        i = PlanInfo()
        _check(lib().pad_plan_get_info(self._h, ctypes.byref(i)))
        return {f: getattr(i, f) for f, _ in PlanInfo._fields_}

    def destroy(self):
        if self._h is not None and _lib is not None:
            _lib.pad_plan_destroy(self._h)
            self._h = None

    def __del__(self):
        self.destroy()


def pad_workspace_size(problem: Problem, prefix_len, event_video) -> int:
    pl, plp = _i32(prefix_len)
    ev, evp = _i32(event_video)
    return int(lib().pad_workspace_size(ctypes.byref(problem), int(pl.size), plp, int(ev.size), evp))


def pad_plan(problem: Problem, cache: CacheState, prefix_len, event_video, event_len,
             page_table=None, max_pages: int = 0, workspace=None, prefix_offset=None,
             stream=None) -> Plan:
    """Plan one decode step (host).  page_table / workspace are device tensors
    (int32 [E, max_pages] / uint8 [bytes]); workspace=None plans on the host only."""
    pl, plp = _i32(prefix_len)
    ev, evp = _i32(event_video)
    el, elp = _i32(event_len)
    po = None
    if prefix_offset is not None:
        po_arr = np.ascontiguousarray(prefix_offset, dtype=np.int64)
        po = po_arr.ctypes.data_as(_I64P)
    if page_table is not None and max_pages == 0:
        max_pages = int(page_table.shape[-1])
    ws_ptr = _ptr(workspace)
    ws_bytes = int(workspace.numel() * workspace.element_size()) if workspace is not None else 0
    strm = _stream(stream) if workspace is not None else c_void_p(0)
    h = c_void_p()
    _check(lib().pad_plan(ctypes.byref(problem), cache.handle, int(pl.size), plp, po, int(ev.size),
                          evp, elp, _ptr(page_table), int(max_pages), ws_ptr, ws_bytes, strm,
                          ctypes.byref(h)))
    return Plan(h, int(el.size))


def pad_kv_append(plan: Plan, k_new, v_new, k_pool, v_pool, stream=None):
    _check(lib().pad_kv_append(plan.handle, _ptr(k_new), _ptr(v_new), _ptr(k_pool), _ptr(v_pool),
                               _stream(stream)))


def pad_event_decode_attn(plan: Plan, q, k_prefix, v_prefix, k_pool, v_pool, out, lse=None,
                          stream=None):
    _check(lib().pad_event_decode_attn(plan.handle, _ptr(q), _ptr(k_prefix), _ptr(v_prefix),
                                       _ptr(k_pool), _ptr(v_pool), _ptr(out), _ptr(lse),
                                       _stream(stream)))


def pad_decode_step(plan: Plan, q, k_new, v_new, k_prefix, v_prefix, k_pool, v_pool, out, lse=None,
                    stream=None):
    """pad_kv_append + pad_event_decode_attn in one call (one kernel launch fewer)."""
    _check(lib().pad_decode_step(plan.handle, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(k_prefix),
                                 _ptr(v_prefix), _ptr(k_pool), _ptr(v_pool), _ptr(out), _ptr(lse),
                                 _stream(stream)))


def pad_prefill_attn(problem, prefix_len: int, branch_len, q, k, v, out, lse=None, stream=None):
    """Whole-sequence forward attention under the event-factorized mask (training / prefill)."""
    bl, blp = _host(branch_len, np.int32)
    _check(lib().pad_prefill_attn(ctypes.byref(problem), int(prefix_len), int(bl.size), blp,
                                  _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), _stream(stream)))


def pad_prefill_status(stream=None):
    """Status word of the last tensor-core prefill launch (synchronises the stream)."""
    _check(lib().pad_prefill_status(_stream(stream)))


def pad_ground_pool(f_proj, offsets, seg_sum, stream=None):
    """Per-segment sums of the projected prefix features (Sec. 3.3 grounding readout)."""
    off, offp = _host(offsets, np.int32)
    _check(lib().pad_ground_pool(_ptr(f_proj), int(f_proj.shape[0]), int(f_proj.shape[1]), offp,
                                 int(off.size - 1), _ptr(seg_sum), _stream(stream)))


def pad_ground_score(g_proj, seg_sum, fraction, scores, salient, interval, stream=None):
    """Segment scores, salient segments and grounded interval of every event token."""
    _check(lib().pad_ground_score(_ptr(g_proj), int(g_proj.shape[0]), _ptr(seg_sum), int(seg_sum.shape[0]),
                                  int(seg_sum.shape[1]), float(fraction), _ptr(scores), _ptr(salient),
                                  _ptr(interval), _stream(stream)))


def aggregate_workspace(n_tokens, n_segments, d_model, device="cuda"):
    """Scratch for pad_attn_aggregate (pad_attn_aggregate_workspace_size bytes of fp32)."""
    import torch
    n = int(lib().pad_attn_aggregate_workspace_size(int(n_tokens), int(n_segments), int(d_model)))
    return torch.empty(max(1, n // 4), dtype=torch.float32, device=device)


def pad_attn_aggregate(x, attn, offsets, interval, g_emb, out, seg_ws, stream=None):
    """Attention-guided pooling of each event's grounded tokens, added to its embedding
    (seg_ws: aggregate_workspace(n_tokens, n_segments, d_model))."""
    off, offp = _host(offsets, np.int32)
    _check(lib().pad_attn_aggregate(_ptr(x), int(x.shape[0]), int(x.shape[1]), _ptr(attn),
                                    offp, int(off.size - 1), _ptr(interval),
                                    int(g_emb.shape[0]), _ptr(g_emb), _ptr(seg_ws),
                                    int(seg_ws.numel() * seg_ws.element_size()), _ptr(out), _stream(stream)))


def pad_event_decode_attn_static(plan: Plan, q, k_prefix, v_prefix, k_pool, v_pool, out, lse=None,
                                 stream=None):
    """pad_event_decode_attn with the library's static scratch instead of a workspace."""
    _check(lib().pad_event_decode_attn_static(plan.handle, _ptr(q), _ptr(k_prefix), _ptr(v_prefix),
                                              _ptr(k_pool), _ptr(v_pool), _ptr(out), _ptr(lse),
                                              _stream(stream)))


def pad_device_status(plan: Plan, stream=None):
    _check(lib().pad_device_status(plan.handle, _stream(stream)))


def _on_gpu(t, name):
    if not t.is_cuda and not t.is_pinned():
        raise ValueError(f"{name}: tensors passed to libpad must be in device memory (or page-locked)")


def _dev(t, name, shape, dtype):
    """Device address of a contiguous tensor of this shape and type (None -> NULL)."""
    if t is None:
        return None
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype}, expected {tuple(shape)} {dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: tensors passed to libpad must be contiguous")
    _on_gpu(t, name)
    return t.data_ptr()


def _rows(t, name, shape, dtype):
    """Device address and row stride (elements; 0 = packed) of a tensor whose rows are contiguous."""
    if t.shape != shape or t.dtype is not dtype:
        raise ValueError(f"{name}: {tuple(t.shape)} {t.dtype}, expected {tuple(shape)} {dtype}")
    _on_gpu(t, name)
    if t.is_contiguous():
        return t.data_ptr(), 0
    want = 1
    for n, st in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if n != 1 and st != want:
            raise ValueError(f"{name}: the rows of tensors passed to libpad must be contiguous")
        want *= n
    if t.shape[0] <= 1:
        return t.data_ptr(), 0
    if t.stride(0) < want:  # (a broadcast one's is 0, which the library takes for packed rows)
        raise ValueError(f"{name}: the rows of tensors passed to libpad must not overlap (row stride {t.stride(0)}, {want} elements)")
    return t.data_ptr(), int(t.stride(0))


class ChunkPlan:
    """A planned step of several tokens per branch (pad_chunk_t)."""

    def __init__(self, handle, problem, n_events, kv_format, n_pages, keep):
        self._h = handle
        self.problem = problem
        self.n_events = n_events
        self.kv_format = kv_format
        self.n_pages = n_pages
        self._keep = keep  # device memory that the plan points to
        i = self.info()
        self.n_tokens, self.n_cached, self.n_drafts = i["n_tokens"], i["n_cached"], i["n_drafts"]
        self._prefix_tokens = i["prefix_tokens"]
        # what every call's tensors are checked against
        import torch
        hq, hk, d = problem.h_q, problem.h_kv, problem.head_dim
        self._q_shape, self._lse_shape = (self.n_tokens, hq, d), (self.n_tokens, hq)
        self._row_shape, self._event_shape, self._params_shape = (self.n_tokens,), (n_events,), (n_events, 4)
        self._new_shape, self._read_shape = (self.n_tokens, hk, d), (self.n_cached, hk, d)
        self._scale_shape = (n_pages, hk, problem.page_size) + ((d // 16,) if kv_format == KV_FP4 else ())
        self._pool_shape = (n_pages, hk, problem.page_size, d // 2 if kv_format == KV_FP4 else d)
        self._bf16, self._f32, self._i32, self._u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
        self._pool_type = torch.bfloat16 if kv_format == KV_BF16 else torch.uint8
        self._out_type = torch.bfloat16 if problem.out_dtype == 1 else torch.float32

    @property
    def handle(self):
        return self._h

    def info(self) -> dict:
        i = ChunkInfo()
        _check(lib().pad_chunk_get_info(self._h, ctypes.byref(i)))
        return {f: getattr(i, f) for f, _ in ChunkInfo._fields_}

    def new_pages(self):
        """(event, column, page) of every page the plan took."""
        n = self.info()["n_new_pages"]
        out = np.zeros((3, n), dtype=np.int32)
        _check(lib().pad_chunk_new_pages(self._h, *(row.ctypes.data_as(_I32P) for row in out)))
        return out[0], out[1], out[2]

    def commit(self, cache, accepted=None) -> np.ndarray:
        """The branches' lengths after verification (pad_chunk_commit); pages past them go back to ``cache``."""
        out = np.zeros(self.n_events, dtype=np.int32)
        acc = accp = None
        if accepted is not None:
            acc, accp = _i32(accepted)
            if acc.size != self.n_events:
                raise ValueError(f"accepted has {acc.size} entries, the plan {self.n_events} events")
        _check(lib().pad_chunk_commit(self._h, None if cache is None else cache.handle, accp,
                                      out.ctypes.data_as(_I32P)))
        return out

    def _pools(self, k_pool, v_pool, k_scale, v_scale):
        ps, pt = self._pool_shape, self._pool_type
        if (k_pool.shape == ps and v_pool.shape == ps and k_pool.dtype is pt and v_pool.dtype is pt
                and k_pool.is_contiguous() and k_pool.is_cuda and v_pool.is_contiguous() and v_pool.is_cuda):
            if k_scale is None and v_scale is None:
                return k_pool.data_ptr(), v_pool.data_ptr(), None, None
            ss, u8 = self._scale_shape, self._u8
            if (k_scale is not None and v_scale is not None and k_scale.shape == ss and v_scale.shape == ss
                    and k_scale.dtype is u8 and v_scale.dtype is u8 and k_scale.is_contiguous() and k_scale.is_cuda
                    and v_scale.is_contiguous() and v_scale.is_cuda):
                return k_pool.data_ptr(), v_pool.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr()
        return (_dev(k_pool, "k_pool", ps, pt), _dev(v_pool, "v_pool", ps, pt),
                _dev(k_scale, "k_scale", self._scale_shape, self._u8), _dev(v_scale, "v_scale", self._scale_shape, self._u8))

    def destroy(self):
        if self._h is not None and _lib is not None:
            _lib.pad_chunk_destroy(self._h)
            self._h = None

    def __del__(self):
        self.destroy()


def _batch(prefix_len, event_video, event_len, n_new):
    el, elp = _i32(event_len)
    nn, nnp = _i32(n_new)
    if el.size != nn.size:
        raise ValueError(f"event_len has {el.size} entries, n_new {nn.size}")
    if prefix_len is None:
        return 0, None, None, el.size, elp, nnp, (el, nn)
    pl, plp = _i32(prefix_len)
    ev, evp = _i32(event_video)
    if ev.size != el.size:
        raise ValueError(f"event_video has {ev.size} entries, event_len {el.size}")
    return int(pl.size), plp, evp, int(el.size), elp, nnp, (el, nn, pl, ev)


def pad_chunk_workspace_size(problem: Problem, prefix_len, event_video, event_len, n_new, kv_format=KV_BF16) -> int:
    nv, plp, evp, ne, elp, nnp, _keep = _batch(prefix_len, event_video, event_len, n_new)
    n = int(lib().pad_chunk_workspace_size(ctypes.byref(problem), int(kv_format), nv, plp, ne, evp, elp, nnp))
    if n == 0:
        raise PadError(1, lib().pad_last_error().decode(errors="replace"))
    return n


def pad_chunk_plan(problem: Problem, cache, prefix_len, event_video, event_len, n_new, page_table=None,
                   n_pages: int = 0, kv_format=KV_BF16, workspace=None, prefix_offset=None, stream=None) -> ChunkPlan:
    """Plan a step of n_new[e] tokens per branch (host, and one copy of the work lists to the workspace).
    ``cache`` None: page_table already lists every page.  ``prefix_len`` None: no prefixes.  workspace=None
    plans on the host only."""
    nv, plp, evp, ne, elp, nnp, _keep = _batch(prefix_len, event_video, event_len, n_new)
    po = None
    if prefix_offset is not None:
        po_arr = np.ascontiguousarray(prefix_offset, dtype=np.int64)
        po = po_arr.ctypes.data_as(_I64P)
    max_pages = 0
    if page_table is not None:
        import torch
        if page_table.dim() != 2 or page_table.shape[0] != ne or page_table.dtype != torch.int32:
            raise ValueError(f"page_table: {tuple(page_table.shape)} {page_table.dtype}, expected [{ne}, max_pages] int32")
        max_pages = int(page_table.shape[1])
    if cache is not None and n_pages == 0:
        n_pages = cache.n_pages
    if workspace is not None:
        _on_gpu(workspace, "workspace")
        if page_table is not None:
            _on_gpu(page_table, "page_table")
    ws_bytes = int(workspace.numel() * workspace.element_size()) if workspace is not None else 0
    strm = _stream(stream) if workspace is not None else c_void_p(0)
    h = c_void_p()
    _check(lib().pad_chunk_plan(ctypes.byref(problem), int(kv_format), None if cache is None else cache.handle, nv, plp,
                                po, ne, evp, elp, nnp, _ptr(page_table), max_pages, int(n_pages), _ptr(workspace),
                                ws_bytes, strm, ctypes.byref(h)))
    return ChunkPlan(h, problem, ne, int(kv_format), int(n_pages), (page_table, workspace))


# (The per-layer calls check their tensors in line, by attribute: a helper call for each would be a quarter of a
# small call's time on the host.  What does not pass goes through the helpers, which say why.)


def pad_chunk_append(plan: ChunkPlan, k_new, v_new, k_pool, v_pool, k_scale=None, v_scale=None, stream=None):
    """Write the new tokens' K/V into the branches' pages (quantised in an 8-bit or 4-bit cache)."""
    shape, bf16 = plan._new_shape, plan._bf16
    if (k_new.shape == shape and v_new.shape == shape and k_new.dtype is bf16 and v_new.dtype is bf16
            and k_new.is_contiguous() and k_new.is_cuda and v_new.is_contiguous() and v_new.is_cuda):
        kn, vn, ks = k_new.data_ptr(), v_new.data_ptr(), 0
    else:
        kn, ks = _rows(k_new, "k_new", shape, bf16)
        vn, vs = _rows(v_new, "v_new", shape, bf16)
        if ks != vs:
            raise ValueError("k_new and v_new must have the same token stride")
    kp, vp, ksc, vsc = plan._pools(k_pool, v_pool, k_scale, v_scale)
    st = (_lib or lib()).pad_chunk_append(plan._h, kn, vn, ks, kp, vp, ksc, vsc, _stream_handle(stream))
    if st:
        _check(st)


class Rope:
    """A model's rotary positions (pad_rope_init): the first ``rotary_dim`` dimensions of a head in pairs (i, i + rotary_dim / 2)
    ("half") or (2 i, 2 i + 1) ("interleaved"), turned by position * theta^(-2 i / rotary_dim).  ``scaling`` for contexts longer than
    the trained ones: "none", "linear", "base", "turns" or "index" (see pad.h for their formulas and what each reads)."""

    LAYOUTS = ("half", "interleaved")
    SCALINGS = ("none", "linear", "base", "turns", "index")

    def __init__(self, head_dim, rotary_dim=None, theta=10000.0, layout="half", scaling="none", factor=1.0, original_len=0.0, low=1.0,
                 high=4.0, magnitude=1.0):
        if layout not in self.LAYOUTS:
            raise ValueError(f"layout {layout!r}, expected one of {self.LAYOUTS}")
        if scaling not in self.SCALINGS:
            raise ValueError(f"scaling {scaling!r}, expected one of {self.SCALINGS}")
        spec = RopeSpec(int(head_dim), int(head_dim if rotary_dim is None else rotary_dim), self.LAYOUTS.index(layout),
                        self.SCALINGS.index(scaling), theta, factor, original_len, low, high, magnitude)
        self.turns = RopeTurns()
        _check(lib().pad_rope_init(ctypes.byref(spec), ctypes.byref(self.turns)))
        self._ref = ctypes.byref(self.turns)


def pad_chunk_append_rope(plan: ChunkPlan, rope: Rope, position, q, q_out, k_new, v_new, k_pool, v_pool, k_scale=None, v_scale=None,
                          stream=None):
    """pad_chunk_append with rotary positions: k_new is turned on its way into the pools, q into q_out (which may be q itself).
    ``position`` [N] int32: of each new token."""
    shape, qs, bf16 = plan._new_shape, plan._q_shape, plan._bf16
    if (k_new.shape == shape and v_new.shape == shape and k_new.dtype is bf16 and v_new.dtype is bf16
            and k_new.is_contiguous() and k_new.is_cuda and v_new.is_contiguous() and v_new.is_cuda):
        kn, vn, ks = k_new.data_ptr(), v_new.data_ptr(), 0
    else:
        kn, ks = _rows(k_new, "k_new", shape, bf16)
        vn, vs = _rows(v_new, "v_new", shape, bf16)
        if ks != vs:
            raise ValueError("k_new and v_new must have the same token stride")
    if (q.shape == qs and q_out.shape == qs and q.dtype is bf16 and q_out.dtype is bf16 and q.is_contiguous() and q.is_cuda
            and q_out.is_contiguous() and q_out.is_cuda):
        qp, op, qst, ost = q.data_ptr(), q_out.data_ptr(), 0, 0
    else:
        qp, qst = _rows(q, "q", qs, bf16)
        op, ost = _rows(q_out, "q_out", qs, bf16)
    if not (position.shape == plan._row_shape and position.dtype is plan._i32 and position.is_contiguous() and position.is_cuda):
        _dev(position, "position", plan._row_shape, plan._i32)
    kp, vp, ksc, vsc = plan._pools(k_pool, v_pool, k_scale, v_scale)
    st = (_lib or lib()).pad_chunk_append_rope(plan._h, rope._ref, position.data_ptr(), qp, qst, op, ost, kn, vn, ks, kp, vp, ksc, vsc,
                                               _stream_handle(stream))
    if st:
        _check(st)


def pad_chunk_read(plan: ChunkPlan, k_pool, v_pool, k_out, v_out, k_scale=None, v_scale=None, stream=None):
    """Copy every branch's cached tokens out as contiguous bf16 [n_cached, h_kv, head_dim]."""
    kp, vp, ksc, vsc = plan._pools(k_pool, v_pool, k_scale, v_scale)
    shape, bf16 = plan._read_shape, plan._bf16
    if not (k_out.shape == shape and v_out.shape == shape and k_out.dtype is bf16 and v_out.dtype is bf16
            and k_out.is_contiguous() and k_out.is_cuda and v_out.is_contiguous() and v_out.is_cuda):
        _dev(k_out, "k_out", shape, bf16)
        _dev(v_out, "v_out", shape, bf16)
    st = (_lib or lib()).pad_chunk_read(plan._h, kp, vp, ksc, vsc, k_out.data_ptr(), v_out.data_ptr(), _stream_handle(stream))
    if st:
        _check(st)


def pad_chunk_attn(plan: ChunkPlan, q, k_prefix, v_prefix, k_pool, v_pool, out, lse=None, k_scale=None, v_scale=None,
                   stream=None):
    """Attention of the step's new tokens over their video's prefix and their branch's cached tokens."""
    shape = plan._q_shape
    if q.shape == shape and q.dtype is plan._bf16 and q.is_contiguous() and q.is_cuda:
        qp, qs = q.data_ptr(), 0
    else:
        qp, qs = _rows(q, "q", shape, plan._bf16)
    if not (out.shape == shape and out.dtype is plan._out_type and out.is_contiguous() and out.is_cuda):
        _dev(out, "out", shape, plan._out_type)
    if lse is None:
        lp = None
    else:
        if not (lse.shape == plan._lse_shape and lse.dtype is plan._f32 and lse.is_contiguous() and lse.is_cuda):
            _dev(lse, "lse", plan._lse_shape, plan._f32)
        lp = lse.data_ptr()
    kp, vp, ksc, vsc = plan._pools(k_pool, v_pool, k_scale, v_scale)
    kx, vx = None, None
    if k_prefix is not None:
        shape, bf16 = k_prefix.shape, plan._bf16
        if shape[0] < plan._prefix_tokens:
            raise ValueError(f"k_prefix: {shape[0]} tokens, the plan reads {plan._prefix_tokens}")
        if not (v_prefix is not None and shape[1:] == plan._new_shape[1:] and v_prefix.shape == shape and k_prefix.dtype is bf16
                and v_prefix.dtype is bf16 and k_prefix.is_contiguous() and k_prefix.is_cuda and v_prefix.is_contiguous() and v_prefix.is_cuda):
            _dev(k_prefix, "k_prefix", (shape[0],) + plan._new_shape[1:], bf16)
            _dev(v_prefix, "v_prefix", shape, bf16)
        kx, vx = k_prefix.data_ptr(), _ptr(v_prefix)
    st = (_lib or lib()).pad_chunk_attn(plan._h, qp, qs, kx, vx, kp, vp, ksc, vsc, out.data_ptr(), lp,
                                        _stream_handle(stream))
    if st:
        _check(st)


def pad_chunk_probs(plan: ChunkPlan, logits, p, params=None, history=None, history_len=None, tokens=None, bias_token=None,
                    bias_value=None, bias_len=None, mask=None, stream=None):
    """The step's logits [n_tokens, vocab] (fp32 or bf16) turned into the probabilities p (fp32 or bf16; may be logits itself) that
    pad_draft_verify reads.  ``params`` [n_events, 4] fp32: temperature, repetition, frequency, presence.  ``history``
    [n_events, width] int32 with ``history_len`` [n_events], ``tokens`` [n_tokens] int32: what counts as repeated.  ``bias_token``
    int32 and ``bias_value`` fp32 [n_events, width] with ``bias_len`` [n_events].  ``mask`` [n_tokens, ceil(vocab / 32)] int32 words."""
    f32, i32, n, ne = plan._f32, plan._i32, plan.n_tokens, plan.n_events
    if logits.dim() != 2:
        raise ValueError(f"logits: {tuple(logits.shape)}, expected [{n}, vocab]")
    shape = (n, logits.shape[1])
    lk, pk = (plan._bf16 if t.dtype is plan._bf16 else f32 for t in (logits, p))
    if (logits.shape == shape and p.shape == shape and logits.dtype is lk and p.dtype is pk and logits.is_contiguous()
            and logits.is_cuda and p.is_contiguous() and p.is_cuda):
        lp, pp, ls, ps = logits.data_ptr(), p.data_ptr(), 0, 0
    else:
        lp, ls = _rows(logits, "logits", shape, lk)
        pp, ps = _rows(p, "p", shape, pk)
    hw = bw = ms = 0
    pa = to = hp = hl = bt = bv = bl = mp = None
    if params is not None:
        if not (params.shape == plan._params_shape and params.dtype is f32 and params.is_contiguous() and params.is_cuda):
            _dev(params, "params", plan._params_shape, f32)
        pa = params.data_ptr()
    if tokens is not None:
        if not (tokens.shape == plan._row_shape and tokens.dtype is i32 and tokens.is_contiguous() and tokens.is_cuda):
            _dev(tokens, "tokens", plan._row_shape, i32)
        to = tokens.data_ptr()
    if history is not None or history_len is not None:
        if history is None or history_len is None:
            raise ValueError("history and history_len come together")
        hw = history.shape[-1]
        if not (history.shape == (ne, hw) and history_len.shape == plan._event_shape
                and history.dtype is i32 and history_len.dtype is i32 and history.is_contiguous() and history.is_cuda
                and history_len.is_contiguous() and history_len.is_cuda):
            _dev(history, "history", (ne, hw), i32), _dev(history_len, "history_len", plan._event_shape, i32)
        if hw:
            hp, hl = history.data_ptr(), history_len.data_ptr()
    if bias_token is not None or bias_value is not None or bias_len is not None:
        if bias_token is None or bias_value is None or bias_len is None:
            raise ValueError("bias_token, bias_value and bias_len come together")
        bw = bias_token.shape[-1]
        bt, bv = _dev(bias_token, "bias_token", (ne, bw), i32), _dev(bias_value, "bias_value", (ne, bw), f32)
        bl = _dev(bias_len, "bias_len", plan._event_shape, i32)
        if not bw:
            bt = bv = bl = None
    if mask is not None:
        mp, ms = _rows(mask, "mask", (n, -(-shape[1] // 32)), i32)
    st = (_lib or lib()).pad_chunk_probs(plan._h, shape[1], 1 if lk is plan._bf16 else 0, lp, ls, pa, to, hp, hw, hl, bt, bv, bw, bl, mp, ms,
                                         1 if pk is plan._bf16 else 0, pp, ps, _stream_handle(stream))
    if st:
        _check(st)


def pad_draft_verify(plan: ChunkPlan, p, q, draft, u_accept, u_pick, accepted, token, stream=None):
    """Accept or reject the step's drafted tokens against the target's probabilities p [n_tokens, vocab] and
    the draft's q [n_drafts, vocab] (fp32 or bf16), and draw each branch's next token."""
    bf16 = p.dtype is plan._bf16
    kind = plan._bf16 if bf16 else plan._f32
    vocab = p.shape[1]
    p_shape, q_shape, nd, ne = (plan.n_tokens, vocab), (plan.n_drafts, vocab), (plan.n_drafts,), (plan.n_events,)
    if (p.shape == p_shape and q.shape == q_shape and p.dtype is kind and q.dtype is kind and p.is_contiguous() and p.is_cuda
            and q.is_contiguous() and q.is_cuda):
        pp, qp, ps, qs = p.data_ptr(), q.data_ptr(), 0, 0
    else:
        pp, ps = _rows(p, "p", p_shape, kind)
        qp, qs = _rows(q, "q", q_shape, kind)
    i32, f32 = plan._i32, plan._f32
    if not (draft.shape == nd and u_accept.shape == nd and u_pick.shape == ne and accepted.shape == ne
            and token.shape == ne and draft.dtype is i32 and u_accept.dtype is f32 and u_pick.dtype is f32
            and accepted.dtype is i32 and token.dtype is i32 and draft.is_contiguous() and draft.is_cuda
            and u_accept.is_contiguous() and u_accept.is_cuda and u_pick.is_contiguous() and u_pick.is_cuda
            and accepted.is_contiguous() and accepted.is_cuda and token.is_contiguous() and token.is_cuda):
        for t, name, shape, dt in ((draft, "draft", nd, i32), (u_accept, "u_accept", nd, f32),
                                   (u_pick, "u_pick", ne, f32), (accepted, "accepted", ne, i32), (token, "token", ne, i32)):
            _dev(t, name, shape, dt)
    st = (_lib or lib()).pad_draft_verify(plan._h, vocab, 1 if bf16 else 0, pp, ps, qp, qs, draft.data_ptr(),
                                          u_accept.data_ptr(), u_pick.data_ptr(), accepted.data_ptr(),
                                          token.data_ptr(), _stream_handle(stream))
    if st:
        _check(st)


def pad_chunk_status(plan: ChunkPlan, stream=None):
    _check(lib().pad_chunk_status(plan.handle, _stream(stream)))


def pad_timing_enable(max_launches: int):
    _check(lib().pad_timing_enable(int(max_launches)))


def pad_timing_read():
    ms = c_float()
    n = c_int32()
    _check(lib().pad_timing_read(ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)


STEP_TWO_CALL = 0x1
STEP_RELEASE_PAGES = 0x2
STEP_MAPPED_HOST_IO = 0x4


class NativeStep:
    """The library's step executor (pad_step_*): every argument marshalled once in C, so a
    step is one call (``run``), or one call with the host copies and the wait included
    (``run_host``).  ``event_len`` is borrowed: update it in place between runs (a
    generation loop), the next run plans from its current values."""

    def __init__(self, problem: Problem, cache: CacheState, prefix_len, event_video, event_len,
                 page_table, max_pages, workspace, prefix_offset, q, k_new, v_new, k_prefix,
                 v_prefix, k_pool, v_pool, out, lse, stream, release_pages=True, one_call=True,
                 rope=None, self_g=None, causal=False, mapped_host_io=False):
        self.L = lib()
        self.problem = problem
        self.cache = cache
        self.prefix_len = np.ascontiguousarray(prefix_len, dtype=np.int32)
        self.event_video = np.ascontiguousarray(event_video, dtype=np.int32)
        # the executor reads this array at every run
        self.event_len = np.array(event_len, dtype=np.int32, copy=True)
        self.prefix_offset = (None if prefix_offset is None
                              else np.ascontiguousarray(prefix_offset, dtype=np.int64))
        self._keep = [q, k_new, v_new, k_prefix, v_prefix, k_pool, v_pool, out, lse, workspace, page_table]
        self.ne = int(self.event_video.size)
        opts = ((0 if one_call else STEP_TWO_CALL) | (STEP_RELEASE_PAGES if release_pages else 0)
                | (STEP_MAPPED_HOST_IO if mapped_host_io else 0))
        h = c_void_p()
        _check(self.L.pad_step_create(
            ctypes.byref(problem), cache.handle, int(self.prefix_len.size), self.prefix_len.ctypes.data_as(_I32P),
            None if self.prefix_offset is None else self.prefix_offset.ctypes.data_as(_I64P), self.ne,
            self.event_video.ctypes.data_as(_I32P), self.event_len.ctypes.data_as(_I32P), _ptr(page_table),
            int(max_pages), _ptr(workspace), int(workspace.numel() * workspace.element_size()), _ptr(q),
            _ptr(k_new), _ptr(v_new), _ptr(k_prefix), _ptr(v_prefix), _ptr(k_pool), _ptr(v_pool), _ptr(out),
            _ptr(lse), _stream(stream), opts, ctypes.byref(h)))
        self.handle = h
        if rope is not None:
            self.rope_pos = np.ascontiguousarray(rope[0], dtype=np.int32)
            self._keep.append(rope[1])
            _check(self.L.pad_step_set_rope(h, self.rope_pos.ctypes.data_as(_I32P), _ptr(rope[1]),
                                            int(rope[1].shape[0])))
        if self_g is not None:
            self.g_k = np.ascontiguousarray(self_g[0], dtype=np.int32)
            self.g_i = np.ascontiguousarray(self_g[1], dtype=np.int32)
            _check(self.L.pad_step_set_g_visibility(h, G_SELF, self.g_k.ctypes.data_as(_I32P),
                                                    self.g_i.ctypes.data_as(_I32P)))
        if causal:
            _check(self.L.pad_step_set_branch_visibility(h, BRANCH_CAUSAL))
        self.new_page = np.full(self.ne, -1, dtype=np.int32)
        self._np = self.new_page.ctypes.data_as(_I32P)
        self._run = self.L.pad_step_run
        self._run_host = self.L.pad_step_run_host

    def __call__(self):
        _check(self._run(self.handle, self._np))

    def run_host(self, h_q, h_k_new, h_v_new, h_out, h_lse=None):
        """Host tensors (page-locked): copies in, the step, copies out, stream wait (with
        mapped_host_io, the inputs are read and the outputs written by kernels over the host
        link where every buffer is page-locked and device-mapped)."""
        _check(self._run_host(self.handle, h_q.data_ptr(), h_k_new.data_ptr(), h_v_new.data_ptr(), h_out.data_ptr(),
                              None if h_lse is None else h_lse.data_ptr(), self._np))

    def enqueue_host(self, h_q, h_k_new, h_v_new, h_out, h_lse=None):
        """run_host without the wait: the buffers stay in use until wait()."""
        _check(self.L.pad_step_enqueue_host(self.handle, h_q.data_ptr(), h_k_new.data_ptr(), h_v_new.data_ptr(),
                                            h_out.data_ptr(), None if h_lse is None else h_lse.data_ptr(),
                                            self._np))

    def wait(self):
        _check(self.L.pad_step_wait(self.handle))

    PROFILE_KEYS = ("host_h2d_call", "host_plan", "host_launch", "host_d2h_call", "host_wait",
                    "host_total", "dev_h2d", "dev_idle_until_launch", "dev_kernels", "dev_d2h",
                    "dev_span")

    def profile(self, enable=True):
        """Per-phase timing of run_host (pad_step_profile); read it with profile_read."""
        _check(self.L.pad_step_profile(self.handle, 1 if enable else 0))

    def profile_read(self):
        buf = (ctypes.c_double * 12)()
        _check(self.L.pad_step_profile_read(self.handle, buf, 12))
        d = dict(zip(self.PROFILE_KEYS, list(buf)[1:]))
        d["calls"] = int(buf[0])
        return d

    def __del__(self):
        h = getattr(self, "handle", None)
        if h is not None and h.value:
            self.L.pad_step_destroy(h)
            self.handle = None
