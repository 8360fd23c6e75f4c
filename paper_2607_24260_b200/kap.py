"""Thin Python binding of the C ABI in include/kap.h - argument marshalling only.

Host-side calls take numpy arrays; the attention calls take torch CUDA tensors (PyTorch is used
for device memory and streams only) and pass raw device pointers and the current CUDA stream.
The shared library must have been built (``python -m paper_2607_24260_b200.build`` or
``__graft_entry__.build()``); there is no fallback path: a missing library raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

from . import build as _build

OK, ERR_INVALID_ARG, ERR_CAPACITY, ERR_UNSUPPORTED, ERR_CUDA, ERR_TIMEOUT, ERR_DEVICE_INDEX = range(7)
PLAN_FULL, PLAN_OVER_BUDGET, PLAN_S_HIGH, PLAN_MOVES_WITH_LENGTH = 1, 2, 4, 8
KV_HND, KV_NHD = 0, 1
LOGITS_F32, LOGITS_BF16 = 0, 1
NORM_F32, NORM_BF16 = 0, 1

_i32p, _f32p, _u8p, _vp = C.POINTER(C.c_int32), C.POINTER(C.c_float), C.POINTER(C.c_uint8), C.c_void_p

# every symbol include/kap.h declares, with its signature
SIGNATURES = {
    "kap_compile_plan": (C.c_int, [C.c_int32, C.c_int32, _i32p, _i32p, _i32p, _i32p, _f32p, _i32p,
                                   _i32p, _i32p, _u8p, C.c_float, _i32p, _i32p, C.c_int64, _i32p,
                                   _i32p, _i32p, _i32p, _i32p, C.POINTER(C.c_uint16)]),
    "kap_compile_growing_plan": (C.c_int, [C.c_int32, C.c_int32, _i32p, _i32p, _i32p, _i32p, _f32p,
                                           _i32p, _i32p, _i32p, _u8p, C.c_float, _i32p, _i32p,
                                           C.c_int32, C.c_int64, _i32p, _i32p, _i32p,
                                           C.POINTER(C.c_uint16), _i32p, _i32p, _i32p]),
    "kap_refresh_recent": (C.c_int, [_vp, _vp, _vp, _vp, _vp, _vp, _vp, _vp, C.c_int32, C.c_int32,
                                     C.c_int64, _vp, _vp, _vp]),
    "kap_workspace_create": (C.c_int, [C.POINTER(_vp), C.c_int32, C.c_int32, C.c_int32, C.c_int32]),
    "kap_workspace_destroy": (None, [_vp]),
    "kap_schedule": (C.c_int, [_vp, C.c_int32, _i32p, _i32p, C.c_int32, C.c_int32, C.c_int32, _vp]),
    "kap_schedule_host": (C.c_int, [C.c_int32, _i32p, _i32p, C.c_int32, C.c_int32, C.c_int32,
                                    C.c_int32, C.c_int32, C.c_int32, _i32p, _i32p, _i32p, _i32p,
                                    _i32p]),
    "kap_schedule_info": (C.c_int, [_vp, _i32p, _i32p, _i32p, _i32p, _i32p]),
    "kap_selected_decode_attn": (C.c_int, [_vp, _vp, C.c_int64, _vp, _vp, _vp, _vp, _vp, C.c_int32,
                                           C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                           _vp, _vp, _vp, _vp]),
    "kap_verify_attn": (C.c_int, [_vp, _vp, _vp, C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32,
                                  C.c_int32, C.c_int32, C.c_int32, C.c_float, _vp, _vp, _vp, _vp]),
    "kap_selected_decode_attn_static": (C.c_int, [_vp, _vp, C.c_int64, _vp, _vp, _vp, _vp, C.c_int32,
                                                  C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                                  C.c_float, C.c_int32, _vp, _vp, _vp, _vp]),
    "kap_append_kv": (C.c_int, [_vp, _vp, _vp, _vp, C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32,
                                C.c_int32, C.c_int32, C.c_int32, C.c_int32, _vp, _vp]),
    "kap_workspace_set_kv_layout": (C.c_int, [_vp, C.c_int32]),
    "kap_top3_accept": (C.c_int, [_vp, C.c_int64, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, _vp, _vp,
                                  _vp, _vp, _vp]),
    "kap_phase_model": (C.c_int, [C.c_double] * 6 + [C.POINTER(C.c_double)]),
    "kap_fallback_decide": (C.c_int, [C.c_int32, C.POINTER(C.c_int64), C.POINTER(C.c_int64), C.c_int64,
                                      C.c_double, C.POINTER(C.c_double), C.POINTER(C.c_double),
                                      C.c_double, C.c_double, C.c_double, C.c_double, _i32p, _i32p,
                                      C.POINTER(C.c_double), C.c_double, _u8p, _i32p,
                                      C.POINTER(C.c_double), C.POINTER(C.c_double),
                                      C.POINTER(C.c_double)]),
    "kap_materialize_view": (C.c_int, [_vp, C.c_int64, _vp, C.c_int64, C.c_int32, C.c_int32, C.c_int32,
                                       _vp, C.c_int64, _vp, _vp, _vp]),
    "kap_append_kv_rope": (C.c_int, [_vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int32,
                                     _vp, C.c_int32, C.c_int32, _vp, C.c_int64, C.c_int32, _vp, _vp, _vp,
                                     C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                     C.c_int32, C.c_int32, C.c_int32, _vp, _vp]),
    "kap_build_block_tables": (C.c_int, [_vp, _vp, _vp, C.c_int32, C.c_int32, _vp, C.c_int32, C.c_int64, _vp, _vp, C.c_int32, _vp,
                                         _vp, _vp, C.c_int64, _vp, _vp, _vp, C.c_int64, _vp, _vp]),
    "kap_release_pages": (C.c_int, [_vp, C.c_int32, _vp, C.c_int32, _vp, C.c_int32, C.c_int64, _vp, _vp, C.c_int32, _vp, _vp, _vp]),
    "kap_adjust_logits": (C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int32, C.c_int32, _vp, C.c_int64, _vp, C.c_int64, _vp, _vp, _vp, _vp,
                                    _vp, _vp, _vp, C.c_int64, _vp, C.c_int32, C.c_int64, _vp, _vp, _vp]),
    "kap_append_kv_norm_rope": (C.c_int, [_vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int64, _vp, C.c_int32,
                                          _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_float,
                                          _vp, C.c_int32, C.c_int32, _vp, C.c_int64, C.c_int32, _vp, _vp, _vp,
                                          C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                          C.c_int32, C.c_int32, C.c_int32, _vp, _vp]),
    "kap_shared_prefix_items": (C.c_int, [C.c_int32, _i32p, _i32p, C.c_int32, _i32p, _i32p, C.c_int32,
                                          C.c_int32, C.c_int32, C.c_int32, _i32p]),
    "kap_schedule_shared_prefix": (C.c_int, [_vp, C.c_int32, _i32p, _i32p, C.c_int32, _i32p, _i32p, C.c_int32,
                                             C.c_int32, _vp]),
    "kap_shared_prefix_attn": (C.c_int, [_vp, _vp, _vp, C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32,
                                         C.c_int32, C.c_int32, C.c_int32, C.c_float, _vp, _vp, _vp, _vp]),
    "kap_chunk_attn_items": (C.c_int, [C.c_int32, C.c_int32, _i32p]),
    "kap_chunk_attn": (C.c_int, [_vp, _vp, C.c_int32, _vp, C.c_int64, _vp, _vp, _vp, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                 C.c_int32, C.c_float, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp]),
    "kap_sample_tokens": (C.c_int, [_vp, C.c_int32, C.c_int64, C.c_int32, C.c_int32, _vp, _vp, _vp, _vp, _vp,
                                    _vp, _vp, _vp]),
    "kap_device_sm_rates": (C.c_int, [C.c_int32, C.c_int32, _f32p, _i32p]),
    "kap_workspace_check": (C.c_int, [_vp, _vp]),
    "kap_set_launch_options": (C.c_int, [C.c_int32] * 5),
    "kap_set_verify_kernel": (C.c_int, [C.c_int32]),
    "kap_launch_count": (C.c_int64, []),
    "kap_last_error": (C.c_char_p, []),
    "kap_version": (C.c_char_p, []),
}

_lib = None


class KapError(RuntimeError):
    def __init__(self, code, message):
        super().__init__(f"kap status {code}: {message}")
        self.code = code


def lib():
    """Load libkap_b200.so (built in-tree).  Raises if it is missing: there is no fallback."""
    global _lib
    if _lib is None:
        path = _build.LIB
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: build it with `python -m paper_2607_24260_b200.build`")
        handle = C.CDLL(path)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype, fn.argtypes = res, args
        _lib = handle
    return _lib


def _check(code):
    if code != OK:
        raise KapError(code, lib().kap_last_error().decode())


def _np(a, dt):
    return None if a is None else np.ascontiguousarray(a, dtype=dt)


def _ptr(a, ct):
    return None if a is None else a.ctypes.data_as(C.POINTER(ct))


def version() -> str:
    return lib().kap_version().decode()


def launch_count() -> int:
    return int(lib().kap_launch_count())


def set_launch_options(use_pdl: int = -1, early_kv: int = -1, ctas_per_sm: int = -1,
                       max_cluster: int = -1, ring_slots: int = -1):
    _check(lib().kap_set_launch_options(int(use_pdl), int(early_kv), int(ctas_per_sm),
                                        int(max_cluster), int(ring_slots)))


def set_verify_kernel(kernel: int):
    """kap_set_verify_kernel: 0 = the mma.sync split kernel, 1 = the tcgen05 kernel (schedules made
    afterwards; at most 64 query rows per KV head, else the split kernel is used)."""
    _check(lib().kap_set_verify_kernel(int(kernel)))


# ------------------------------------------------------------------------------- kap_compile_plan
def compile_plan(ctx_len, span_indptr, span_start, span_len, span_score, budget_tokens, n_sink,
                 n_recent, force_full=None, s_max=1.0, bt_indptr=None, bt_pages=None, page_size=16,
                 capacity=None):
    """kap_compile_plan on host arrays.  Returns a dict: plan_indptr, plan_logical_pages,
    plan_phys_pages (None without a block table), plan_flags, selected_tokens, plan_token_masks
    (uint16 per listed page, bit t = token t of the page is in the selected union; None when
    page_size > 16)."""
    ctx_len = _np(ctx_len, np.int32)
    B = int(ctx_len.shape[0])
    span_indptr, span_start = _np(span_indptr, np.int32), _np(span_start, np.int32)
    span_len, span_score = _np(span_len, np.int32), _np(span_score, np.float32)
    budget_tokens, n_sink = _np(budget_tokens, np.int32), _np(n_sink, np.int32)
    n_recent, force_full = _np(n_recent, np.int32), _np(force_full, np.uint8)
    bt_indptr, bt_pages = _np(bt_indptr, np.int32), _np(bt_pages, np.int32)
    if capacity is None:
        capacity = int(sum((max(int(L), 0) + page_size - 1) // max(page_size, 1) for L in ctx_len))
    indptr = np.full(B + 1, -1, dtype=np.int32)
    logical = np.full(max(1, capacity), -1, dtype=np.int32)
    phys = np.full(max(1, capacity), -1, dtype=np.int32) if bt_indptr is not None else None
    flags = np.full(B, -1, dtype=np.int32)
    sel = np.full(B, -1, dtype=np.int32)
    masks = np.zeros(max(1, capacity), dtype=np.uint16) if 0 < page_size <= 16 else None
    _check(lib().kap_compile_plan(
        B, page_size, _ptr(ctx_len, C.c_int32), _ptr(span_indptr, C.c_int32),
        _ptr(span_start, C.c_int32), _ptr(span_len, C.c_int32), _ptr(span_score, C.c_float),
        _ptr(budget_tokens, C.c_int32), _ptr(n_sink, C.c_int32), _ptr(n_recent, C.c_int32),
        _ptr(force_full, C.c_uint8), float(s_max), _ptr(bt_indptr, C.c_int32),
        _ptr(bt_pages, C.c_int32), int(capacity), _ptr(indptr, C.c_int32), _ptr(logical, C.c_int32),
        _ptr(phys, C.c_int32), _ptr(flags, C.c_int32), _ptr(sel, C.c_int32),
        _ptr(masks, C.c_uint16)))
    n = int(indptr[-1])
    return dict(plan_indptr=indptr, plan_logical_pages=logical[:n].copy(),
                plan_phys_pages=None if phys is None else phys[:n].copy(), plan_flags=flags,
                selected_tokens=sel,
                plan_token_masks=None if masks is None else masks[:n].copy())


def compile_growing_plan(ctx_len, span_indptr, span_start, span_len, span_score, budget_tokens,
                         n_sink, n_recent, bt_indptr, bt_pages, force_full=None, s_max=1.0,
                         page_size=16, max_growth=0, capacity=None):
    """kap_compile_growing_plan on host arrays.  Returns the dict of compile_plan (lists = fixed
    part + reserved entries) plus tail_desc int32 [B, 3]."""
    ctx_len = _np(ctx_len, np.int32)
    B = int(ctx_len.shape[0])
    span_indptr, span_start = _np(span_indptr, np.int32), _np(span_start, np.int32)
    span_len, span_score = _np(span_len, np.int32), _np(span_score, np.float32)
    budget_tokens, n_sink = _np(budget_tokens, np.int32), _np(n_sink, np.int32)
    n_recent, force_full = _np(n_recent, np.int32), _np(force_full, np.uint8)
    bt_indptr, bt_pages = _np(bt_indptr, np.int32), _np(bt_pages, np.int32)
    if capacity is None:
        ps = max(page_size, 1)
        capacity = int(sum((max(int(L), 0) + ps - 1) // ps + (max(int(r), 1) + ps - 2) // ps + 1
                           + (max_growth + ps - 1) // ps + 1 for L, r in zip(ctx_len, n_recent)))
    indptr = np.full(B + 1, -1, dtype=np.int32)
    logical = np.full(max(1, capacity), -1, dtype=np.int32)
    phys = np.full(max(1, capacity), -1, dtype=np.int32)
    masks = np.zeros(max(1, capacity), dtype=np.uint16)
    flags = np.full(B, -1, dtype=np.int32)
    sel = np.full(B, -1, dtype=np.int32)
    tail = np.full((B, 3), -1, dtype=np.int32)
    _check(lib().kap_compile_growing_plan(
        B, page_size, _ptr(ctx_len, C.c_int32), _ptr(span_indptr, C.c_int32),
        _ptr(span_start, C.c_int32), _ptr(span_len, C.c_int32), _ptr(span_score, C.c_float),
        _ptr(budget_tokens, C.c_int32), _ptr(n_sink, C.c_int32), _ptr(n_recent, C.c_int32),
        _ptr(force_full, C.c_uint8), float(s_max), _ptr(bt_indptr, C.c_int32),
        _ptr(bt_pages, C.c_int32), int(max_growth), int(capacity), _ptr(indptr, C.c_int32),
        _ptr(logical, C.c_int32), _ptr(phys, C.c_int32), _ptr(masks, C.c_uint16),
        _ptr(flags, C.c_int32), _ptr(sel, C.c_int32), _ptr(tail, C.c_int32)))
    n = int(indptr[-1])
    return dict(plan_indptr=indptr, plan_logical_pages=logical[:n].copy(),
                plan_phys_pages=phys[:n].copy(), plan_flags=flags, selected_tokens=sel,
                plan_token_masks=masks[:n].copy(), tail_desc=tail)


def refresh_recent(plan_indptr, plan_logical_pages, plan_phys_pages, plan_token_masks, tail_desc,
                   bt_indptr, bt_pages, ctx_len, num_pool_pages, ws: "Workspace | None" = None,
                   device_status=None, page_size=16, stream=None):
    """kap_refresh_recent on torch CUDA tensors (int32; masks as 16-bit words): rewrites the
    reserved entries of a growing plan from the current device ctx_len."""
    _check(lib().kap_refresh_recent(
        _dptr(plan_indptr), _dptr(plan_logical_pages), _dptr(plan_phys_pages),
        _dptr(plan_token_masks), _dptr(tail_desc), _dptr(bt_indptr), _dptr(bt_pages),
        _dptr(ctx_len), int(ctx_len.shape[0]), int(page_size), int(num_pool_pages),
        _dptr(device_status), None if ws is None else ws._h, _stream_ptr(stream)))


def compile_workload(w, capacity=None):
    """kap_compile_plan on a synth.Workload."""
    return compile_plan(w.ctx_len, w.span_indptr, w.span_start, w.span_len, w.span_score,
                        w.budget_tokens, w.n_sink, w.n_recent, w.force_full, w.s_max, w.bt_indptr,
                        w.bt_pages, w.page_size, capacity)


def schedule_host(list_len, n_q, num_q_heads, num_kv_heads, cta_slots, max_chunk_pages=0,
                  max_items=8192, max_cluster=1):
    """kap_schedule_host: the split-K work list as an [n_items, 8] int32 array (seq, kv_head,
    page_begin, page_end, group, slot, n_splits, n_q) plus (n_merge_groups, max_chunk) and, when
    max_cluster > 1, the chosen cluster size as a fourth value."""
    list_len = _np(list_len, np.int32)
    n_q = _np(n_q, np.int32)
    items = np.zeros((max_items, 8), dtype=np.int32)
    n_items, n_merge, max_chunk, cluster = C.c_int32(0), C.c_int32(0), C.c_int32(0), C.c_int32(1)
    _check(lib().kap_schedule_host(int(list_len.shape[0]), _ptr(list_len, C.c_int32),
                                   _ptr(n_q, C.c_int32), num_q_heads, num_kv_heads, cta_slots,
                                   max_cluster, max_chunk_pages, max_items, _ptr(items, C.c_int32),
                                   C.byref(n_items), C.byref(n_merge), C.byref(max_chunk),
                                   C.byref(cluster)))
    out = (items[:n_items.value].copy(), n_merge.value, max_chunk.value)
    return out if max_cluster <= 1 else out + (cluster.value,)


# ------------------------------------------------------------------------- workspace + attention
_torch = _BF16 = _F32 = _I32 = _current_stream = None


def _torch_module():
    global _torch, _BF16, _F32, _I32, _current_stream
    if _torch is None:
        import torch
        _BF16, _F32, _I32 = torch.bfloat16, torch.float32, torch.int32
        _current_stream = _stream_reader(torch)
        _torch = torch
    return _torch


def _stream_reader(torch):
    """the handle of a device's current stream: read without building a Stream object for it (4 us less a call), where torch offers that"""
    return getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda dev: torch.cuda.current_stream(dev).cuda_stream)


def _stream_ptr(stream=None):
    """the handle of a torch stream, or of the current one"""
    if stream is not None:
        return stream.cuda_stream
    torch = _torch_module()
    return _current_stream(torch.cuda.current_device())


def _stream_on(dev, stream):
    """_stream_ptr for tensors on device dev: kernels are launched on the current device, so they have to be there"""
    current = _torch.cuda.current_device()
    if dev != current:
        raise KapError(ERR_INVALID_ARG, f"the tensors are on device {dev}, but device {current} is current")
    return _current_stream(dev) if stream is None else stream.cuda_stream


def _dptr(t):
    return None if t is None else t.data_ptr()


def _pool_shape(kv_pool, ws):
    """(pages, Hkv, P) of a pool tensor in the layout the workspace is set to"""
    pages, _, a, b, _ = kv_pool.shape
    return (pages, b, a) if getattr(ws, "kv_layout", KV_HND) == KV_NHD else (pages, a, b)


def _dense_pool(kv_pool, nhd, dev):
    """(pages, Hkv, P, d) of a pool tensor that the kernels can address"""
    shape = kv_pool.shape
    if kv_pool.dtype is not _BF16 or shape[1] != 2 or not kv_pool.is_contiguous() or kv_pool.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"kv_pool is {kv_pool.dtype} {tuple(shape)} with strides {kv_pool.stride()} on {kv_pool.device}, "
                       f"expected a contiguous bfloat16 tensor of K and V on GPU {dev}")
    pages, _, a, b, d = shape
    return (pages, b, a, d) if nhd else (pages, a, b, d)


def _check_index(name, t, least, dev):
    if t.dtype is not _I32 or t.get_device() != dev or not t.is_contiguous() or t.numel() < least:
        raise KapError(ERR_INVALID_ARG, f"{name} is {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}, expected a "
                       f"contiguous int32 tensor of at least {least} on GPU {dev}")


def _check_block_table(bt_indptr, bt_pages, ctx_len, batch, dev):
    if bt_indptr.dtype is not _I32 or bt_pages.dtype is not _I32 or ctx_len.dtype is not _I32 or bt_indptr.numel() <= batch or \
            bt_indptr.get_device() != dev or bt_pages.get_device() != dev or ctx_len.get_device() != dev or \
            not bt_indptr.is_contiguous() or not bt_pages.is_contiguous() or not ctx_len.is_contiguous():
        _check_index("bt_indptr", bt_indptr, batch + 1, dev)
        _check_index("bt_pages", bt_pages, 0, dev)
        _check_index("ctx_len", ctx_len, batch, dev)


class Workspace:
    """kap_workspace: split-K schedule + partial-result buffers for one launch shape."""

    def __init__(self, device=0, max_items=8192, max_rows_per_item=16, max_batch=256):
        self._h = C.c_void_p()
        self.device = int(device)
        self.kv_layout = KV_HND
        self.shared_prefix_rows = 0          # of the last schedule_shared_prefix
        self._destroy = lib().kap_workspace_destroy
        _check(lib().kap_workspace_create(C.byref(self._h), self.device, max_items,
                                          max_rows_per_item, max_batch))

    def close(self):
        if getattr(self, "_h", None) is not None and self._h:
            self._destroy(self._h)           # bound at construction: module globals may be gone at exit
            self._h = None

    __del__ = close

    def schedule(self, list_len, n_q=None, num_q_heads=32, num_kv_heads=8, max_chunk_pages=0,
                 stream=None):
        list_len = _np(list_len, np.int32)
        n_q = _np(n_q, np.int32)
        _check(lib().kap_schedule(self._h, int(list_len.shape[0]), _ptr(list_len, C.c_int32),
                                  _ptr(n_q, C.c_int32), num_q_heads, num_kv_heads, max_chunk_pages,
                                  _stream_ptr(stream)))
        return self.info()

    def set_kv_layout(self, kv_layout):
        """KV_HND (default): pools are [pages, 2, Hkv, P, d]; KV_NHD: [pages, 2, P, Hkv, d]."""
        _check(lib().kap_workspace_set_kv_layout(self._h, int(kv_layout)))
        self.kv_layout = int(kv_layout)

    def schedule_shared_prefix(self, list_len, n_q, group_indptr, prefix_pages, num_q_heads=32,
                               num_kv_heads=8, stream=None):
        """kap_schedule_shared_prefix on host arrays (see kap.h); shared_prefix_items gives the
        max_items the workspace needs."""
        list_len, n_q = _np(list_len, np.int32), _np(n_q, np.int32)
        group_indptr, prefix_pages = _np(group_indptr, np.int32), _np(prefix_pages, np.int32)
        _check_groups(list_len, n_q, group_indptr, prefix_pages)
        _check(lib().kap_schedule_shared_prefix(
            self._h, int(list_len.shape[0]), _ptr(list_len, C.c_int32), _ptr(n_q, C.c_int32),
            int(prefix_pages.shape[0]), _ptr(group_indptr, C.c_int32), _ptr(prefix_pages, C.c_int32),
            num_q_heads, num_kv_heads, _stream_ptr(stream)))
        self.shared_prefix_rows = int(n_q.sum())

    def info(self):
        v = [C.c_int32(0) for _ in range(5)]
        _check(lib().kap_schedule_info(self._h, *[C.byref(x) for x in v]))
        return dict(n_items=v[0].value, n_merge_groups=v[1].value, max_chunk_pages=v[2].value,
                    ctas_per_wave=v[3].value, cluster_size=v[4].value)

    def check(self, stream=None):
        _check(lib().kap_workspace_check(self._h, _stream_ptr(stream)))


def selected_decode_attn(q, kv_pool, plan_indptr, plan_phys_pages, plan_logical_pages, ctx_len, out,
                         ws: Workspace, lse=None, sm_scale=None, stream=None, plan_token_masks=None):
    """kap_selected_decode_attn on torch CUDA tensors: q/out bf16 [B, Hq, d]; kv_pool bf16
    [pages, 2, Hkv, P, d]; plan arrays and ctx_len int32 device tensors; plan_token_masks an
    optional uint16 device tensor (one word per listed page) for token-granular visibility."""
    B, Hq, d = q.shape
    pages, Hkv, P = _pool_shape(kv_pool, ws)
    sm_scale = float(d) ** -0.5 if sm_scale is None else float(sm_scale)
    _check(lib().kap_selected_decode_attn(
        _dptr(q), _dptr(kv_pool), int(pages), _dptr(plan_indptr), _dptr(plan_phys_pages),
        _dptr(plan_logical_pages), _dptr(plan_token_masks), _dptr(ctx_len), B, Hq, Hkv, d, P,
        sm_scale, _dptr(out), _dptr(lse), ws._h, _stream_ptr(stream)))
    return out


def verify_attn(q, q_indptr, kv_pool, bt_indptr, bt_pages, ctx_len, out, ws: Workspace, lse=None,
                sm_scale=None, stream=None):
    """kap_verify_attn on torch CUDA tensors: q/out bf16 [sum n_q, Hq, d]."""
    _, Hq, d = q.shape
    pages, Hkv, P = _pool_shape(kv_pool, ws)
    sm_scale = float(d) ** -0.5 if sm_scale is None else float(sm_scale)
    _check(lib().kap_verify_attn(
        _dptr(q), _dptr(q_indptr), _dptr(kv_pool), int(pages), _dptr(bt_indptr), _dptr(bt_pages),
        _dptr(ctx_len), int(ctx_len.shape[0]), Hq, Hkv, d, P, sm_scale, _dptr(out), _dptr(lse),
        ws._h, _stream_ptr(stream)))
    return out


def _check_groups(list_len, n_q, group_indptr, prefix_pages):
    if n_q.shape != list_len.shape or group_indptr.shape != (prefix_pages.shape[0] + 1,):
        raise KapError(ERR_INVALID_ARG, f"{list_len.shape[0]} list lengths, {n_q.shape[0]} row counts, "
                       f"{group_indptr.shape[0]} group offsets, {prefix_pages.shape[0]} prefixes")


def shared_prefix_items(list_len, n_q, group_indptr, prefix_pages, num_q_heads=32, num_kv_heads=8,
                        max_rows_per_item=64, cta_slots=148):
    """kap_shared_prefix_items: the max_items of a Workspace (with this max_rows_per_item) that can
    hold the schedule of schedule_shared_prefix on a device of cta_slots SMs."""
    list_len, n_q = _np(list_len, np.int32), _np(n_q, np.int32)
    group_indptr, prefix_pages = _np(group_indptr, np.int32), _np(prefix_pages, np.int32)
    _check_groups(list_len, n_q, group_indptr, prefix_pages)
    n = C.c_int32(0)
    _check(lib().kap_shared_prefix_items(
        int(list_len.shape[0]), _ptr(list_len, C.c_int32), _ptr(n_q, C.c_int32), int(prefix_pages.shape[0]),
        _ptr(group_indptr, C.c_int32), _ptr(prefix_pages, C.c_int32), num_q_heads, num_kv_heads,
        int(max_rows_per_item), int(cta_slots), C.byref(n)))
    return n.value


def shared_prefix_attn(q, q_indptr, kv_pool, bt_indptr, bt_pages, ctx_len, out, ws: Workspace, lse=None,
                       sm_scale=None, stream=None):
    """kap_shared_prefix_attn on torch CUDA tensors: the arguments and the result of verify_attn, for a
    workspace scheduled with schedule_shared_prefix.  q, out and lse have at least the scheduled rows."""
    (rows, Hq, d), (out_rows, out_heads, out_d), need = q.shape, out.shape, ws.shared_prefix_rows
    lse_rows, lse_heads = (need, Hq) if lse is None else lse.shape
    if rows < need or out_rows < need or lse_rows < need or out_heads != Hq or lse_heads != Hq or out_d != d:
        raise KapError(ERR_INVALID_ARG, f"q {tuple(q.shape)}, out {tuple(out.shape)}, lse {None if lse is None else tuple(lse.shape)}: "
                       f"expected at least {need} scheduled rows of {Hq} heads")
    _torch_module()
    dev = ws.device
    if q.dtype is not _BF16 or out.dtype is not _BF16 or not q.is_contiguous() or not out.is_contiguous() or q.get_device() != dev or out.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"q is {q.dtype} with strides {q.stride()} on {q.device}, out {out.dtype} with strides {out.stride()} on "
                       f"{out.device}: expected contiguous bfloat16 tensors on GPU {dev}, the workspace's device")
    if lse is not None and (lse.dtype is not _F32 or not lse.is_contiguous() or lse.get_device() != dev):
        raise KapError(ERR_INVALID_ARG, f"lse is {lse.dtype} with strides {lse.stride()} on {lse.device}, expected a contiguous float32 tensor on GPU {dev}")
    batch = ctx_len.shape[0]
    _check_index("q_indptr", q_indptr, batch + 1, dev)
    _check_block_table(bt_indptr, bt_pages, ctx_len, batch, dev)
    pages, Hkv, P, pool_d = _dense_pool(kv_pool, ws.kv_layout == KV_NHD, dev)
    if pool_d != d:
        raise KapError(ERR_INVALID_ARG, f"q has heads of {d} columns, kv_pool of {pool_d}")
    sm_scale = d ** -0.5 if sm_scale is None else float(sm_scale)
    _check(lib().kap_shared_prefix_attn(
        q.data_ptr(), q_indptr.data_ptr(), kv_pool.data_ptr(), pages, bt_indptr.data_ptr(), bt_pages.data_ptr(),
        ctx_len.data_ptr(), batch, Hq, Hkv, d, P, sm_scale, out.data_ptr(), _dptr(lse),
        ws._h, _stream_on(dev, stream)))
    return out


def chunk_attn_items(max_rows_per_item=64, cta_slots=148):
    """kap_chunk_attn_items: the max_items of a Workspace (with this max_rows_per_item) that can hold the
    partial results of chunk_attn on a device of cta_slots SMs."""
    n = C.c_int32(0)
    _check(lib().kap_chunk_attn_items(int(max_rows_per_item), int(cta_slots), C.byref(n)))
    return n.value


def chunk_attn(q, q_indptr, kv_pool, bt_indptr, bt_pages, ctx_len, out, ws: Workspace, lse=None, window=0,
               n_sink=0, sm_scale=None, stream=None):
    """kap_chunk_attn on torch CUDA tensors: q/out bf16 [rows, Hq, d], the rows of sequence b at
    q_indptr[b] .. q_indptr[b+1]-1; window 0 sees the whole context, otherwise the last `window` tokens and
    the first n_sink.  The workspace needs no schedule, only the size that chunk_attn_items gives."""
    _torch_module()
    dev = ws.device
    if q.dtype is not _BF16 or out.dtype is not _BF16 or q.dim() != 3 or out.shape != q.shape or not q.is_contiguous() or \
            not out.is_contiguous() or q.get_device() != dev or out.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"q is {q.dtype} {tuple(q.shape)} with strides {q.stride()} on {q.device}, out {out.dtype} {tuple(out.shape)} with "
                       f"strides {out.stride()} on {out.device}: expected contiguous bfloat16 tensors of one shape on GPU {dev}, the workspace's device")
    rows, Hq, d = q.shape
    if lse is not None and (lse.dtype is not _F32 or lse.shape != (rows, Hq) or not lse.is_contiguous() or lse.get_device() != dev):
        raise KapError(ERR_INVALID_ARG, f"lse is {lse.dtype} {tuple(lse.shape)} with strides {lse.stride()} on {lse.device}, expected a contiguous "
                       f"float32 [{rows}, {Hq}] tensor on GPU {dev}")
    batch = ctx_len.shape[0]
    _check_index("q_indptr", q_indptr, batch + 1, dev)
    _check_block_table(bt_indptr, bt_pages, ctx_len, batch, dev)
    pages, Hkv, P, pool_d = _dense_pool(kv_pool, ws.kv_layout == KV_NHD, dev)
    if pool_d != d:
        raise KapError(ERR_INVALID_ARG, f"q has heads of {d} columns, kv_pool of {pool_d}")
    sm_scale = d ** -0.5 if sm_scale is None else float(sm_scale)
    _check(lib().kap_chunk_attn(
        q.data_ptr(), q_indptr.data_ptr(), rows, kv_pool.data_ptr(), pages, bt_indptr.data_ptr(), bt_pages.data_ptr(),
        ctx_len.data_ptr(), batch, Hq, Hkv, d, P, sm_scale, window, n_sink, out.data_ptr(), _dptr(lse),
        ws._h, _stream_on(dev, stream)))
    return out


def selected_decode_attn_static(q, kv_pool, plan_indptr, plan_phys_pages, plan_logical_pages, ctx_len,
                                out, num_splits, lse=None, device_status=None, sm_scale=None,
                                stream=None):
    """kap_selected_decode_attn_static: the proposal-path attention without a workspace, for
    callers that may not allocate device memory (scratch is a fixed array inside the library).
    `device_status`: optional int32 CUDA tensor of one element that receives the status bits."""
    B, Hq, d = q.shape
    pages, _, Hkv, P, _ = kv_pool.shape
    sm_scale = float(d) ** -0.5 if sm_scale is None else float(sm_scale)
    _check(lib().kap_selected_decode_attn_static(
        _dptr(q), _dptr(kv_pool), int(pages), _dptr(plan_indptr), _dptr(plan_phys_pages),
        _dptr(plan_logical_pages), _dptr(ctx_len), B, Hq, Hkv, d, P, sm_scale, int(num_splits),
        _dptr(out), _dptr(lse), _dptr(device_status), _stream_ptr(stream)))
    return out


def append_kv(k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, new_indptr=None, advance=True,
              device_status=None, stream=None, kv_layout=KV_HND):
    """kap_append_kv: write the new tokens' K/V rows (bf16 [sum n_new, Hkv, d]) into the paged pool
    at positions ctx_len[b] .. and, with advance, bump ctx_len on the device.  kv_pool has shape
    [pages, 2, Hkv, P, d] (KV_HND) or [pages, 2, P, Hkv, d] (KV_NHD)."""
    if kv_layout == KV_NHD:
        pages, _, P, Hkv, d = kv_pool.shape
    else:
        pages, _, Hkv, P, d = kv_pool.shape
    _check(lib().kap_append_kv(_dptr(k_new), _dptr(v_new), _dptr(new_indptr), _dptr(kv_pool), int(pages),
                               _dptr(bt_indptr), _dptr(bt_pages), _dptr(ctx_len), int(bool(advance)),
                               int(ctx_len.shape[0]), Hkv, d, P, int(kv_layout), _dptr(device_status),
                               _stream_ptr(stream)))


def _page_state(page_table, pages_held, free_pages, free_count):
    """(requests, table_stride, device) of the arrays that build_block_tables and release_pages keep"""
    _torch_module()
    i32, dev, shape = _I32, page_table.get_device(), page_table.shape
    if dev < 0 or len(shape) != 2 or page_table.dtype is not i32 or not page_table.is_contiguous():
        raise KapError(ERR_INVALID_ARG, f"page_table is {page_table.dtype} {tuple(shape)} with strides {page_table.stride()} on "
                       f"{page_table.device}, expected a contiguous int32 [requests, pages] tensor on a GPU")
    requests, wide = shape
    if pages_held.dtype is not i32 or free_pages.dtype is not i32 or free_count.dtype is not i32 or pages_held.get_device() != dev or \
            free_pages.get_device() != dev or free_count.get_device() != dev or not pages_held.is_contiguous() or \
            not free_pages.is_contiguous() or pages_held.numel() < requests or free_count.numel() < 1:
        _check_index("pages_held", pages_held, requests, dev)
        _check_index("free_pages", free_pages, 0, dev)
        _check_index("free_count", free_count, 1, dev)
    return requests, wide, dev


def build_block_tables(ctx_len, page_table, pages_held, free_pages, free_count, bt_indptr, bt_pages, n_new=None, request=None,
                       new_indptr=None, slot=None, position=None, page_size=16, device_status=None, stream=None):
    """kap_build_block_tables on torch CUDA tensors (int32; slot int64): the CSR block table of the step's sequences
    (request[b], ctx_len[b] tokens cached, n_new[b] new ones; None: row b of page_table, one new token), with the pages it lacks taken
    from free_pages[:free_count].  page_table [requests, pages], pages_held [requests], free_pages and free_count [1] are kept up to
    date (an entry of page_table whose page the caller has put back on the stack itself is negative); new_indptr [batch + 1], slot and position [rows] are optional."""
    requests, wide, dev = _page_state(page_table, pages_held, free_pages, free_count)
    batch, lists = ctx_len.shape[0], bt_pages.numel()
    if ctx_len.dtype is not _I32 or bt_indptr.dtype is not _I32 or bt_pages.dtype is not _I32 or ctx_len.get_device() != dev or \
            bt_indptr.get_device() != dev or bt_pages.get_device() != dev or not ctx_len.is_contiguous() or \
            not bt_indptr.is_contiguous() or not bt_pages.is_contiguous() or bt_indptr.numel() <= batch:
        _check_index("ctx_len", ctx_len, batch, dev)
        _check_index("bt_indptr", bt_indptr, batch + 1, dev)
        _check_index("bt_pages", bt_pages, 0, dev)
    n_new_at = request_at = new_at = slot_at = position_at = status_at = None
    rows = -1
    if n_new is not None:
        _check_index("n_new", n_new, batch, dev)
        n_new_at = n_new.data_ptr()
    if request is not None:
        _check_index("request", request, batch, dev)
        request_at = request.data_ptr()
    if new_indptr is not None:
        _check_index("new_indptr", new_indptr, batch + 1, dev)
        new_at = new_indptr.data_ptr()
    if slot is not None:
        if slot.dtype is not _torch.int64 or slot.get_device() != dev or not slot.is_contiguous():
            raise KapError(ERR_INVALID_ARG, f"slot is {slot.dtype} with strides {slot.stride()} on {slot.device}, expected a contiguous int64 tensor on GPU {dev}")
        slot_at, rows = slot.data_ptr(), slot.numel()
    if position is not None:
        _check_index("position", position, 0, dev)
        position_at, n = position.data_ptr(), position.numel()
        rows = n if rows < 0 or n < rows else rows
    if device_status is not None:
        _check_index("device_status", device_status, 1, dev)
        status_at = device_status.data_ptr()
    _check(lib().kap_build_block_tables(
        request_at, ctx_len.data_ptr(), n_new_at, batch, page_size, page_table.data_ptr(), requests, wide, pages_held.data_ptr(),
        free_pages.data_ptr(), free_pages.numel(), free_count.data_ptr(), bt_indptr.data_ptr(), bt_pages.data_ptr(), lists,
        new_at, slot_at, position_at, max(rows, 0), status_at, _stream_on(dev, stream)))


def release_pages(request, page_table, pages_held, free_pages, free_count, keep_tokens=None, page_size=16, device_status=None,
                  stream=None):
    """kap_release_pages on torch CUDA tensors: the pages of the requests beyond keep_tokens (None: all) go back to the
    stack; negative entries of page_table, whose pages are there already, are passed over.  request None names every row of page_table."""
    requests, wide, dev = _page_state(page_table, pages_held, free_pages, free_count)
    n, request_at, keep_at, status_at = requests, None, None, None
    if request is not None:
        n = request.numel()
        _check_index("request", request, n, dev)
        request_at = request.data_ptr()
    if keep_tokens is not None:
        _check_index("keep_tokens", keep_tokens, n, dev)
        keep_at = keep_tokens.data_ptr()
    if device_status is not None:
        _check_index("device_status", device_status, 1, dev)
        status_at = device_status.data_ptr()
    _check(lib().kap_release_pages(
        request_at, n, keep_at, page_size, page_table.data_ptr(), requests, wide, pages_held.data_ptr(), free_pages.data_ptr(),
        free_pages.numel(), free_count.data_ptr(), status_at, _stream_on(dev, stream)))


def _head_rows(name, t, rows, heads, d, dev):
    """the row stride of a bf16 [rows, heads, d] tensor whose heads are contiguous within a row"""
    if t.dtype is not _BF16 or t.shape != (rows, heads, d) or t.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"{name} is {t.dtype} {tuple(t.shape)} on {t.device}, expected bfloat16 [{rows}, {heads}, {d}] on GPU {dev}")
    if t.is_contiguous():
        return heads * d
    stride = t.stride()
    if stride[2] != 1 or (heads > 1 and stride[1] != d):
        raise KapError(ERR_INVALID_ARG, f"{name} has strides {stride}: the heads of a row must be contiguous")
    return heads * d if rows <= 1 else stride[0]


def append_kv_rope(q, k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, inv_freq, q_out=None,
                   new_indptr=None, positions=None, freq_axis=None, position_offset=None,
                   interleaved=False, advance=True, device_status=None, stream=None, kv_layout=KV_HND):
    """kap_append_kv_rope: rotate q and k_new (bf16 [rows, heads, d], any row stride) by
    position * inv_freq (fp32 [rotary_dim / 2]) and write k and v_new into the paged pool like
    append_kv.  q_out None rotates q in place; q None handles k and v only.  positions None: the
    logical index (+ position_offset[b]); else int32 [rows] or [axes, rows], freq_axis naming the axis
    of each pair (host sequence)."""
    _append_rope(None, q, k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, inv_freq, q_out, new_indptr, positions,
                 freq_axis, position_offset, interleaved, advance, device_status, stream, kv_layout)


def append_kv_norm_rope(q, k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, inv_freq, q_weight=None, k_weight=None,
                        eps=1e-6, unit_offset=False, q_out=None, new_indptr=None, positions=None, freq_axis=None,
                        position_offset=None, interleaved=False, advance=True, device_status=None, stream=None,
                        kv_layout=KV_HND):
    """kap_append_kv_norm_rope: append_kv_rope with the heads of q and k_new normalised before the rotation,
    x / sqrt(mean(x^2) + eps) * weight (1 + weight with unit_offset).  Weights: fp32 or bf16, both of one
    type and form, [d] for all heads or [heads, d]; None means 1."""
    _append_rope((q_weight, k_weight, eps, unit_offset), q, k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, inv_freq, q_out,
                 new_indptr, positions, freq_axis, position_offset, interleaved, advance, device_status, stream, kv_layout)


def _norm_arguments(norm, Hq, Hkv, d, dev):
    """(q_weight, k_weight, type, per head, unit offset, eps) of kap_append_kv_norm_rope"""
    q_weight, k_weight, eps, unit_offset = norm
    if Hq and q_weight is not None and k_weight is not None and q_weight.dtype is k_weight.dtype and (k_weight.dtype is _F32 or k_weight.dtype is _BF16) and \
            q_weight.is_contiguous() and k_weight.is_contiguous() and q_weight.get_device() == dev and k_weight.get_device() == dev:
        shapes, heads = (q_weight.shape, k_weight.shape), 0
        if shapes == ((Hq, d), (Hkv, d)):
            heads = 1
        if heads or shapes == ((d,), (d,)):                       # the usual forms; all others, and what is wrong, below
            return (q_weight.data_ptr(), k_weight.data_ptr(), NORM_F32 if k_weight.dtype is _F32 else NORM_BF16, heads, 1 if unit_offset else 0, eps)
    kinds = set()
    for name, w, heads in (("q_weight", q_weight, Hq), ("k_weight", k_weight, Hkv)):
        if w is None or (name == "q_weight" and Hq == 0):
            continue
        if w.dtype is not _F32 and w.dtype is not _BF16 or w.shape != (d,) and w.shape != (heads, d) or not w.is_contiguous() or w.get_device() != dev:
            raise KapError(ERR_INVALID_ARG, f"{name} is {w.dtype} {tuple(w.shape)} with strides {w.stride()} on {w.device}, expected a contiguous "
                           f"float32 or bfloat16 tensor [{d}] or [{heads}, {d}] on GPU {dev}")
        kinds.add((w.dtype, w.dim()))
    if len(kinds) > 1:
        raise KapError(ERR_INVALID_ARG, f"q_weight and k_weight differ in type or form: {kinds}")
    dtype, dims = kinds.pop() if kinds else (_F32, 1)
    return (_dptr(q_weight) if Hq else None, _dptr(k_weight), NORM_F32 if dtype is _F32 else NORM_BF16, 1 if dims == 2 else 0,
            1 if unit_offset else 0, eps)


def _append_rope(norm, q, k_new, v_new, kv_pool, bt_indptr, bt_pages, ctx_len, inv_freq, q_out, new_indptr, positions, freq_axis,
                 position_offset, interleaved, advance, device_status, stream, kv_layout):
    _torch_module()
    rows, Hq, dev = k_new.shape[0], 0, k_new.get_device()
    if dev < 0:
        raise KapError(ERR_INVALID_ARG, "k_new is not on a GPU")
    pages, Hkv, P, d = _dense_pool(kv_pool, kv_layout == KV_NHD, dev)
    ks, vs = _head_rows("k_new", k_new, rows, Hkv, d, dev), _head_rows("v_new", v_new, rows, Hkv, d, dev)
    qs = os_ = 0
    if q is None:
        q_out = None
    else:
        Hq = q.shape[1]
        qs = _head_rows("q", q, rows, Hq, d, dev)
        if q_out is None:
            q_out, os_ = q, qs
        else:
            os_ = _head_rows("q_out", q_out, rows, Hq, d, dev)
    axes, pos_stride = 0, 0
    if positions is not None:
        if positions.dim() == 1:
            positions = positions.view(1, -1)
        if positions.dtype is not _I32 or positions.shape[1] != rows or (rows > 1 and positions.stride(1) != 1) or positions.get_device() != dev:
            raise KapError(ERR_INVALID_ARG, f"positions {positions.dtype} {tuple(positions.shape)} on {positions.device} for {rows} rows on GPU {dev}")
        axes, pos_stride = positions.shape[0], positions.stride(0)
        if axes == 1:
            pos_stride = max(pos_stride, rows)
    if inv_freq.dtype is not _F32 or not inv_freq.is_contiguous() or inv_freq.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"inv_freq must be a contiguous float32 tensor on GPU {dev}, not {inv_freq.dtype} on {inv_freq.device}")
    rot = 2 * inv_freq.shape[0]
    axis = None
    if freq_axis is not None:
        axis = bytes(freq_axis) if type(freq_axis) in (list, tuple, bytes) else _np(freq_axis, np.uint8).tobytes()
        if len(axis) != rot // 2:
            raise KapError(ERR_INVALID_ARG, f"freq_axis names {len(axis)} pairs, inv_freq {rot // 2}")
    batch = ctx_len.shape[0]
    _check_block_table(bt_indptr, bt_pages, ctx_len, batch, dev)
    if new_indptr is not None:
        _check_index("new_indptr", new_indptr, batch + 1, dev)
    if position_offset is not None:
        _check_index("position_offset", position_offset, batch, dev)
    if device_status is not None:
        _check_index("device_status", device_status, 1, dev)
    middle = () if norm is None else _norm_arguments(norm, Hq, Hkv, d, dev)
    first = (_dptr(q), qs, k_new.data_ptr(), ks, v_new.data_ptr(), vs, _dptr(q_out), os_, _dptr(new_indptr), rows)
    rest = (inv_freq.data_ptr(), rot, 1 if interleaved else 0, _dptr(positions), pos_stride, axes, axis,
            _dptr(position_offset), kv_pool.data_ptr(), pages, bt_indptr.data_ptr(), bt_pages.data_ptr(),
            ctx_len.data_ptr(), 1 if advance else 0, batch, Hq, Hkv, d, P, kv_layout,
            _dptr(device_status), _stream_on(dev, stream))
    if norm is None:
        _check(lib().kap_append_kv_rope(*first, *rest))
    else:
        _check(lib().kap_append_kv_norm_rope(*first, *middle, *rest))


def _array(name, t, dtype, n, dev):
    """the address of a contiguous tensor of n elements (n < 0: any number)"""
    if t.dtype is not dtype or (n >= 0 and t.numel() != n) or not t.is_contiguous() or t.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"{name} is {t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}, expected a contiguous {dtype} "
                       f"tensor{f' of {n}' if n >= 0 else ''} on GPU {dev}")
    return t.data_ptr()


def adjust_logits(logits, out=None, history=None, history_at=None, repetition=None, presence=None, frequency=None, bias_indptr=None,
                  bias_token=None, bias_value=None, allowed=None, allowed_row=None, device_status=None, stream=None):
    """kap_adjust_logits on torch CUDA tensors: logits and out fp32 or bf16 [rows, vocab] (any row stride; out None: in place);
    history int32, history_at int64 [rows, 3] (prompt from, answer from, end); repetition, presence, frequency fp32 [rows]; biases as
    int32 bias_indptr [rows + 1], int32 bias_token, fp32 bias_value; allowed int32 bit masks [masks, words], allowed_row int32 [rows]."""
    _torch_module()
    kind = LOGITS_F32 if logits.dtype is _F32 else LOGITS_BF16 if logits.dtype is _BF16 else None
    if kind is None or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1) or not logits.is_cuda:
        raise KapError(ERR_INVALID_ARG, f"logits are {logits.dtype} {tuple(logits.shape)} with strides {logits.stride()} on {logits.device}")
    (rows, vocab), dev = logits.shape, logits.get_device()
    if out is None:
        out = logits
    elif out.dtype is not logits.dtype or out.shape != logits.shape or (vocab > 1 and out.stride(1) != 1) or out.get_device() != dev:
        raise KapError(ERR_INVALID_ARG, f"out is {out.dtype} {tuple(out.shape)} with strides {out.stride()} on {out.device}, logits {logits.dtype} {tuple(logits.shape)} on GPU {dev}")

    f32, i32 = _F32, _I32
    masks = words = 0
    if allowed is not None:
        if allowed.dim() != 2 or allowed.dtype is not i32 or (allowed.shape[1] > 1 and allowed.stride(1) != 1) or allowed.get_device() != dev:
            raise KapError(ERR_INVALID_ARG, f"allowed is {allowed.dtype} {tuple(allowed.shape)} with strides {allowed.stride()} on {allowed.device}, expected int32 [masks, words]")
        masks, words = allowed.shape[0], allowed.stride(0) if allowed.shape[0] > 1 else allowed.shape[1]
        if allowed.shape[1] * 32 < vocab:
            raise KapError(ERR_INVALID_ARG, f"allowed has {allowed.shape[1]} words for {vocab} logits")
    if (history is None) != (history_at is None):
        raise KapError(ERR_INVALID_ARG, "history and history_at go together")
    if (bias_token is None) != (bias_indptr is None) or (bias_value is None) != (bias_indptr is None):
        raise KapError(ERR_INVALID_ARG, "bias_indptr, bias_token and bias_value go together")
    if bias_token is not None and bias_token.numel() != bias_value.numel():
        raise KapError(ERR_INVALID_ARG, f"{bias_token.numel()} bias tokens, {bias_value.numel()} values")
    wide = vocab if rows <= 1 else logits.stride(0)
    _check(lib().kap_adjust_logits(
        logits.data_ptr(), kind, wide, rows, vocab, out.data_ptr(), wide if out is logits else vocab if rows <= 1 else out.stride(0),
        None if history is None else _array("history", history, i32, -1, dev), 0 if history is None else history.numel(),
        None if history_at is None else _array("history_at", history_at, _torch.int64, 3 * rows, dev),
        None if repetition is None else _array("repetition", repetition, f32, rows, dev),
        None if presence is None else _array("presence", presence, f32, rows, dev),
        None if frequency is None else _array("frequency", frequency, f32, rows, dev),
        None if bias_indptr is None else _array("bias_indptr", bias_indptr, i32, rows + 1, dev),
        None if bias_token is None else _array("bias_token", bias_token, i32, -1, dev),
        None if bias_value is None else _array("bias_value", bias_value, f32, -1, dev), 0 if bias_token is None else bias_token.numel(),
        None if allowed is None else allowed.data_ptr(), masks, words,
        None if allowed_row is None else _array("allowed_row", allowed_row, i32, rows, dev),
        None if device_status is None else _array("device_status", device_status, i32, 1, dev), _stream_on(dev, stream)))
    return out


def sample_tokens(logits, uniform, token, logprob=None, temperature=None, top_k=None, top_p=None,
                  min_p=None, stream=None):
    """kap_sample_tokens on torch CUDA tensors: logits fp32 or bf16 [rows, vocab] (any row stride), uniform
    fp32 [rows]; outputs int32 token [rows] and optional fp32 logprob [rows].  temperature, top_p,
    min_p (fp32 [rows]) and top_k (int32 [rows]) are optional; None switches a filter off."""
    _torch_module()
    kind = LOGITS_F32 if logits.dtype is _F32 else LOGITS_BF16 if logits.dtype is _BF16 else None
    if kind is None or logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1) or not logits.is_cuda:
        raise KapError(ERR_INVALID_ARG, f"logits are {logits.dtype} {tuple(logits.shape)} with strides {logits.stride()} on {logits.device}")
    (rows, vocab), dev = logits.shape, logits.get_device()

    def ptr(name, t, dt):
        if t is None:
            return None
        if t.dtype is not dt or t.numel() != rows or not t.is_contiguous() or t.get_device() != dev:
            raise KapError(ERR_INVALID_ARG, f"{name} must be a contiguous {dt} tensor of {rows} on GPU {dev}")
        return t.data_ptr()

    f32, i32 = _F32, _I32
    _check(lib().kap_sample_tokens(
        logits.data_ptr(), kind, vocab if rows <= 1 else logits.stride(0), rows, vocab,
        ptr("temperature", temperature, f32), ptr("top_k", top_k, i32), ptr("top_p", top_p, f32), ptr("min_p", min_p, f32),
        ptr("uniform", uniform, f32), ptr("token", token, i32), ptr("logprob", logprob, f32), _stream_on(dev, stream)))


def top3_accept(logits, row_indptr, proposed, top3, accepted, next_token, stream=None, ctx_len=None):
    """kap_top3_accept on torch CUDA tensors: logits fp32 [rows, vocab] (row stride taken from the
    tensor), int32 row_indptr [B+1], proposed [rows]; outputs int32 top3 [rows, 3], accepted [B],
    next_token [B].  ctx_len (int32 [B], optional) is reduced by the number of rejected proposals."""
    rows, vocab = logits.shape
    _check(lib().kap_top3_accept(_dptr(logits), int(logits.stride(0)), _dptr(row_indptr), _dptr(proposed),
                                 int(row_indptr.shape[0]) - 1, int(rows), int(vocab), _dptr(top3),
                                 _dptr(accepted), _dptr(next_token), _dptr(ctx_len), _stream_ptr(stream)))


PHASE_FIELDS = ("cost_full", "cost_base", "cost_plan", "speedup", "slack", "kv_crit", "beneficial",
                "h_minus_s")


def phase_model(k, h, s, w_main, w_prop, kv):
    """kap_phase_model: dict of the cost model's quantities (Eqs. 3-15)."""
    out = (C.c_double * 8)()
    _check(lib().kap_phase_model(float(k), float(h), float(s), float(w_main), float(w_prop), float(kv), out))
    return dict(zip(PHASE_FIELDS, [float(x) for x in out]))


FALLBACK_CAPACITY, FALLBACK_METADATA, FALLBACK_CONFIDENCE, FALLBACK_S_HIGH, FALLBACK_H_LOW, \
    FALLBACK_NO_MARGIN, FALLBACK_SLACK = 1, 2, 4, 8, 16, 32, 64
RUNTIME_OVER_CAPACITY, RUNTIME_UNSTABLE_METADATA = 1, 2


def fallback_decide(accepted_sum, proposed_sum, s, kv, w_main=0.0, w_prop=0.0, min_proposed=1,
                    h_prior=1.0, h_min=0.0, s_max=1.0, plan_flags=None, runtime_flags=None,
                    confidence=None, confidence_min=0.0):
    """kap_fallback_decide on host arrays; returns a dict of numpy arrays: force_full (uint8, ready
    for compile_plan's force_full), reasons, h, slack, budget_scale."""
    acc, prop = _np(accepted_sum, np.int64), _np(proposed_sum, np.int64)
    s, kv = _np(s, np.float64), _np(kv, np.float64)
    B = int(s.shape[0])
    flags, rt, conf = _np(plan_flags, np.int32), _np(runtime_flags, np.int32), _np(confidence, np.float64)
    out = dict(force_full=np.zeros(B, dtype=np.uint8), reasons=np.zeros(B, dtype=np.int32),
               h=np.zeros(B), slack=np.zeros(B), budget_scale=np.zeros(B))
    _check(lib().kap_fallback_decide(
        B, _ptr(acc, C.c_int64), _ptr(prop, C.c_int64), int(min_proposed), float(h_prior),
        _ptr(s, C.c_double), _ptr(kv, C.c_double), float(w_main), float(w_prop), float(h_min),
        float(s_max), _ptr(flags, C.c_int32), _ptr(rt, C.c_int32), _ptr(conf, C.c_double),
        float(confidence_min), _ptr(out["force_full"], C.c_uint8), _ptr(out["reasons"], C.c_int32),
        _ptr(out["h"], C.c_double), _ptr(out["slack"], C.c_double), _ptr(out["budget_scale"], C.c_double)))
    return out


def device_sm_rates(device=0):
    """kap_device_sm_rates: numpy array of the relative streaming rate of every SM (mean 1)."""
    n = C.c_int32(0)
    _check(lib().kap_device_sm_rates(int(device), 0, None, C.byref(n)))
    out = np.zeros(n.value, dtype=np.float32)
    _check(lib().kap_device_sm_rates(int(device), n.value, _ptr(out, C.c_float), C.byref(n)))
    return out


def materialize_view(kv_pool, plan_phys_pages, compact_pool, compact_pages=None, device_status=None,
                     stream=None):
    """kap_materialize_view: copy the plan's pages into compact_pool in plan order."""
    pages, _, Hkv, P, d = kv_pool.shape
    _check(lib().kap_materialize_view(_dptr(kv_pool), int(pages), _dptr(plan_phys_pages),
                                      int(plan_phys_pages.shape[0]), Hkv, d, P, _dptr(compact_pool),
                                      int(compact_pool.shape[0]), _dptr(compact_pages),
                                      _dptr(device_status), _stream_ptr(stream)))
