"""Thin ctypes binding over libtokenlake.so: same names as the C ABI (include/tokenlake.h),
argument marshalling only.  Every step of the path runs in the library's kernels; there is
no Python or CPU fallback -- if the library is missing, loading raises.

Device arguments are torch tensors (their data_ptr is passed) or raw integer addresses;
host arrays are numpy arrays.  `stream=None` uses torch's current HIP stream.
"""
from __future__ import annotations

import ctypes as C
import math
import os
from itertools import accumulate, chain
from operator import mul
from struct import Struct
from typing import Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtokenlake.so")

TL_OK, TL_EINVAL, TL_ENOMEM, TL_EFULL, TL_ENOTFOUND, TL_EHIP = 0, -1, -2, -3, -4, -5
TL_PLAN_SELF_BLOCK, TL_PLAN_NO_SHARING, TL_PLAN_FUSE_ROWS, TL_PLAN_WALK_REPEATS, TL_PLAN_FUSE_TAILS = 1, 2, 4, 8, 16


class TokenLakeError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("tokenlake status %d: %s" % (status, message))
        self.status = status


class tl_plan_info(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_req", "n_tokens", "q_heads", "kv_heads", "n_items", "n_partial_rows", "self_row_base",
        "n_tiles", "n_units", "n_causal_tiles", "n_list_entries", "n_merge_entries")] + [
        (n, C.c_int64) for n in ("prefix_pairs", "self_pairs", "unique_kv_tokens")] + [
        (n, C.c_int32) for n in ("n_fused_tiles", "n_fused_tokens", "n_single_tokens")] + [
        ("tile_pairs", C.c_int64), ("item_pairs", C.c_int64), ("n_prior_rows", C.c_int32), ("n_unit_workgroups", C.c_int32)]


class tl_rope(C.Structure):
    _fields_ = [("steps_dev", C.c_void_p), ("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_float)]


class tl_qkv(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v")] + [
        (n, C.c_int64) for n in ("q_row_stride", "q_head_stride", "k_row_stride", "k_head_stride", "v_row_stride", "v_head_stride")] + [
        (n, C.c_int32) for n in ("q_heads", "kv_heads", "is_bf16")] + [("eps", C.c_float)] + [
        (n, C.c_void_p) for n in ("q_weight", "k_weight", "q_out", "k_out", "v_out")]


_lib = None

_P, _I32, _U64, _F32, _F64 = C.c_void_p, C.c_int32, C.c_uint64, C.c_float, C.c_double
_PF64 = C.POINTER(C.c_double)
_SIGNATURES = {
    "tl_status_str": (C.c_char_p, [_I32]),
    "tl_last_error": (C.c_char_p, []),
    "tl_set_option": (_I32, [C.c_char_p, _I32]),
    "tl_pool_create": (_I32, [C.POINTER(_P), _I32, _I32, _I32, _I32, _P, _P]),
    "tl_pool_destroy": (_I32, [_P]),
    "tl_pool_put": (_I32, [_P, _U64, _P, _P, _I32, _I32, C.POINTER(_I32), _P]),
    "tl_pool_append": (_I32, [_P, _I32, _U64, _P, _I32, _P, _P, _I32, _P, _P]),
    "tl_pool_append_batch": (_I32, [_P, _I32, _P, _P, _P, _P, _P, _P, _P, _P, _P]),
    "tl_pool_reserve_batch": (_I32, [_P, _I32, _P, _P, _P, _P, _P, _P, _P]),
    "tl_pool_adopt": (_I32, [_P, _P, _P, _P, _I32, _P]),
    "tl_pool_release": (_I32, [_P, _U64]),
    "tl_pool_evict_lru": (_I32, [_P, C.POINTER(_U64)]),
    "tl_pool_lookup": (_I32, [_P, _P, _I32, _P]),
    "tl_pool_hot_segments": (_I32, [_P, _I32, _P, _P, _P, C.POINTER(_I32)]),
    "tl_pool_prefix_tree": (_I32, [_P, _I32, _P, _P, _P, C.POINTER(_I32), C.POINTER(_I32)]),
    "tl_pool_fills": (_I32, [_P, _P, _I32, _P]),
    "tl_pool_used": (_I32, [_P, C.POINTER(_I32)]),
    "tl_pool_gather": (_I32, [_P, _P, _I32, _P, _P, _P]),
    "tl_plan_create": (_I32, [C.POINTER(_P), _P, _I32, _I32, _P, _P, _P, _I32, _I32, _I32]),
    "tl_plan_destroy": (_I32, [_P]),
    "tl_plan_get_info": (_I32, [_P, C.POINTER(tl_plan_info)]),
    "tl_plan_export_sizes": (_I32, [_P, C.POINTER(_I32), C.POINTER(_I32)]),
    "tl_plan_hot_slots": (_I32, [_P, _I32, _P, _P, C.POINTER(_I32)]),
    "tl_plan_export": (_I32, [_P, _P, _P, _P, _P, _P, _P, _P]),
    "tl_segment_attn": (_I32, [_P, _P, _P, _F32, _P, _P, _P]),
    "tl_causal_block": (_I32, [_P, _P, _P, _P, _F32, _P, _P, _P]),
    "tl_merge": (_I32, [_P, _P, _P, _P, _I32, _P, _P]),
    "tl_fused_attn": (_I32, [_P, _P, _P, _P, _P, _F32, _P, _P, _P, _I32, _P, _P]),
    "tl_fused_attn_static": (_I32, [_P, _P, _P, _P, _P, _F32, _P, _P, _P, _I32, _P, _P]),
    "tl_rope_steps": (_I32, [_P, _I32, _P]),
    "tl_rotate_rows": (_I32, [_P, _P, _P, _I32, _P]),
    "tl_pool_write_rows": (_I32, [_P, _P, _P, _P, _P, _I32, _P]),
    "tl_pool_move_rows": (_I32, [_P, _P, _P, _P, _P, _I32, _P]),
    "tl_model_segment_time": (_I32, [_F64, _F64, _F64, _F64, _F64, _PF64]),
    "tl_model_comm_time": (_I32, [_F64, _F64, _F64, _PF64]),
    "tl_model_segment_threshold": (_I32, [_F64, _F64, _F64, _F64, _F64, _F64, _PF64]),
    "tl_model_cache_load": (_I32, [_F64, _P, _P, _I32, _I32, _F64, _F64, _F64, _PF64, _PF64, _PF64]),
    "tl_segment_ids": (_I32, [_P, C.c_int64, _I32, C.c_uint64, _P]),
}
EXPORTED = tuple(_SIGNATURES)


def load_library(path: Optional[str] = None):
    """Load libtokenlake.so (built by paper_2508_17219_amd.build).  Raises if it is absent."""
    global _lib
    if _lib is None:
        p = path or os.environ.get("TOKENLAKE_LIB") or LIB_PATH
        if not os.path.exists(p):
            raise FileNotFoundError(
                "%s not found: build it with `python -m paper_2508_17219_amd.build` "
                "(there is no fallback path)" % p)
        lib = C.CDLL(p)
        for name, (res, args) in _SIGNATURES.items():
            fn = getattr(lib, name)
            fn.restype, fn.argtypes = res, args
        _lib = lib
    return _lib


def _check(status: int):
    if status != TL_OK:
        raise TokenLakeError(status, load_library().tl_last_error().decode())


def _dev(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if not x.is_contiguous():
        raise ValueError("device tensor must be contiguous")
    return x.data_ptr()


def _host(a, dtype) -> np.ndarray:
    if type(a) is np.ndarray and a.dtype == dtype and a.ndim and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


def _offsets(counts, n: int) -> np.ndarray:
    """0 and the running sums of n counts."""
    # (plain ints alone: narrow numpy scalars would be added in their own width, one-element lists strung together.  Anything else
    # in the list leaves its type in the last sum: looking at every entry's type takes 16 counts 1.03 us, this 0.82)
    if type(counts) is list and n and len(counts) == n and type(counts[0]) is int:
        try:
            sums = [0, *accumulate(counts)]
            if type(sums[-1]) is int:
                return np.array(sums, np.int32)
        except Exception:       # numpy's to take or refuse
            pass
    out = np.zeros(n + 1, np.int32)
    out[1:] = np.cumsum(counts)
    return out


def _addr(a: np.ndarray) -> int:
    """Address of an array's data (`a.ctypes.data` builds an object for it)."""
    return a.__array_interface__["data"][0]


_raw_stream = None      # () -> handle of torch's current stream, once torch can use a GPU


def _stream_getter(torch):
    """torch's own getters where this torch has them: they are not part of its public interface."""
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if raw is None or device is None:
        return lambda: torch.cuda.current_stream().cuda_stream
    return lambda: raw(device())


def _stream(stream) -> Optional[int]:
    """torch's current stream as a handle: asked of torch directly, because a `torch.cuda.Stream` object and the
    availability check in front of it cost 4 us a call, as much as a launch."""
    global _raw_stream
    if stream is None:
        import torch
        if _raw_stream is None:
            if not torch.cuda.is_available():
                return None
            torch.cuda.init()
            _raw_stream = _stream_getter(torch)
        return _raw_stream() or None
    return int(stream) or None


# ---- pool -------------------------------------------------------------------------------
def tl_pool_create(n_slots: int, seg_len: int, kv_heads: int, head_dim: int, k_dev=None, v_dev=None) -> int:
    h = _P()
    _check(load_library().tl_pool_create(C.byref(h), n_slots, seg_len, kv_heads, head_dim, _dev(k_dev), _dev(v_dev)))
    return h.value


def tl_pool_destroy(pool: int):
    _check(load_library().tl_pool_destroy(pool))


def tl_pool_put(pool: int, segment_id: int, k_src, v_src, fill: int, want_slot: int = -1, stream=None) -> int:
    slot = _I32(-1)
    _check(load_library().tl_pool_put(pool, segment_id, _dev(k_src), _dev(v_src), fill, want_slot, C.byref(slot),
                                      _stream(stream)))
    return slot.value


def tl_pool_append(pool: int, tail_id, new_ids, k_rows, v_rows, n_rows: int, stream=None) -> np.ndarray:
    """tail_id None = no partly filled tail.  Returns the slots given to new_ids."""
    ids = _host(new_ids, np.uint64)
    slots = np.full(len(ids), -1, np.int32)
    _check(load_library().tl_pool_append(pool, 0 if tail_id is None else 1, 0 if tail_id is None else int(tail_id),
                                         ids.ctypes.data if len(ids) else None, len(ids), _dev(k_rows), _dev(v_rows),
                                         n_rows, slots.ctypes.data if len(ids) else None, _stream(stream)))
    return slots


def tl_pool_append_batch(pool: int, tail_ids, new_ids, row_counts, k_rows, v_rows, stream=None) -> np.ndarray:
    """One call for many chains.  tail_ids: per chain an id or None; new_ids: per chain a list of
    ids; row_counts: per chain the number of rows it takes from k_rows/v_rows (in chain order).
    Returns the slots given to the new ids, flattened in chain order."""
    # (a serving engine makes this call once per decoded token: running sums of a few entries cost less as Python lists, and
    # so do the arrays' addresses without ctypes, 16 chains 22.8 -> 14.1 us in front of the library's call)
    n = len(tail_ids)
    has_tail = np.array([t is not None for t in tail_ids], np.int32)
    tails = np.array([0 if t is None else int(t) for t in tail_ids], np.uint64)
    new_ptr, row_ptr = _offsets(list(map(len, new_ids)), n), _offsets(row_counts, n)
    ids = np.array(list(chain.from_iterable(new_ids)), np.uint64)
    slots = np.full(len(ids), -1, np.int32)
    has_ids = len(ids) > 0
    _check(load_library().tl_pool_append_batch(pool, n, _addr(has_tail), _addr(tails), _addr(new_ptr), _addr(ids) if has_ids else None,
                                               _addr(row_ptr), _dev(k_rows), _dev(v_rows), _addr(slots) if has_ids else None,
                                               _stream(stream)))
    return slots


def tl_pool_reserve_batch(pool: int, tail_ids, new_ids, row_counts):
    """The arguments of tl_pool_append_batch without the rows.  Returns (slots of the new ids, pool row of each of the chains' rows)."""
    n = len(tail_ids)
    has_tail = np.array([t is not None for t in tail_ids], np.int32)
    tails = np.array([0 if t is None else int(t) for t in tail_ids], np.uint64)
    new_ptr, row_ptr = _offsets(list(map(len, new_ids)), n), _offsets(row_counts, n)
    ids = np.array(list(chain.from_iterable(new_ids)), np.uint64)
    slots, rows = np.full(len(ids), -1, np.int32), np.full(max(int(row_ptr[-1]), 0), -1, np.int32)
    _check(load_library().tl_pool_reserve_batch(pool, n, _addr(has_tail), _addr(tails), _addr(new_ptr), _addr(ids) if len(ids) else None,
                                                _addr(row_ptr), _addr(slots) if len(ids) else None, _addr(rows) if len(rows) else None))
    return slots, rows


def tl_pool_adopt(pool: int, ids, slots, fills, stream=None):
    ids, slots, fills = _host(ids, np.uint64), _host(slots, np.int32), _host(fills, np.int32)
    if not (len(ids) == len(slots) == len(fills)):
        raise ValueError("ids/slots/fills length mismatch")
    _check(load_library().tl_pool_adopt(pool, ids.ctypes.data, slots.ctypes.data, fills.ctypes.data, len(ids),
                                        _stream(stream)))


def tl_pool_release(pool: int, segment_id: int):
    _check(load_library().tl_pool_release(pool, segment_id))


def tl_pool_evict_lru(pool: int) -> int:
    out = _U64(0)
    _check(load_library().tl_pool_evict_lru(pool, C.byref(out)))
    return out.value


def tl_pool_hot_segments(pool: int, max_n: int):
    """(ids, loads, depths) of the prefix tree's most loaded nodes, at most max_n, parents first."""
    m = max(max_n, 1)
    ids, loads, depths, n = np.zeros(m, np.uint64), np.zeros(m, np.int64), np.zeros(m, np.int32), _I32(0)
    _check(load_library().tl_pool_hot_segments(pool, max_n, ids.ctypes.data, loads.ctypes.data, depths.ctypes.data, C.byref(n)))
    return ids[:n.value], loads[:n.value], depths[:n.value]


def tl_pool_prefix_tree(pool: int, max_nodes: int):
    """(ids, parents, loads, n_total): the pool's prefix tree in level order, at most max_nodes nodes."""
    m = max(max_nodes, 1)
    ids, parents, loads = np.zeros(m, np.uint64), np.zeros(m, np.int32), np.zeros(m, np.int64)
    n, total = _I32(0), _I32(0)
    _check(load_library().tl_pool_prefix_tree(pool, max_nodes, ids.ctypes.data, parents.ctypes.data, loads.ctypes.data,
                                              C.byref(n), C.byref(total)))
    return ids[:n.value], parents[:n.value], loads[:n.value], total.value


def tl_pool_lookup(pool: int, ids) -> np.ndarray:
    ids = _host(ids, np.uint64)
    out = np.empty(len(ids), np.int32)
    _check(load_library().tl_pool_lookup(pool, ids.ctypes.data, len(ids), out.ctypes.data))
    return out


def tl_pool_fills(pool: int, slots) -> np.ndarray:
    slots = _host(slots, np.int32)
    out = np.empty(len(slots), np.int32)
    _check(load_library().tl_pool_fills(pool, slots.ctypes.data, len(slots), out.ctypes.data))
    return out


def tl_pool_used(pool: int) -> int:
    n = _I32(0)
    _check(load_library().tl_pool_used(pool, C.byref(n)))
    return n.value


def tl_pool_gather(pool: int, slots, k_out, v_out, stream=None):
    slots = _host(slots, np.int32)
    _check(load_library().tl_pool_gather(pool, slots.ctypes.data, len(slots), _dev(k_out), _dev(v_out), _stream(stream)))


# ---- plan -------------------------------------------------------------------------------
def tl_plan_create(pool: int, q_heads: int, req_row_ptr, req_seg_ptr, seg_ids, flags: int = TL_PLAN_SELF_BLOCK,
                   split_segments: int = 0, compute_units: int = -1) -> int:
    rp, sp, ids = _host(req_row_ptr, np.int32), _host(req_seg_ptr, np.int32), _host(seg_ids, np.uint64)
    if len(rp) != len(sp) or len(rp) < 1:
        raise ValueError("req_row_ptr/req_seg_ptr must both have n_req+1 entries")
    if len(ids) < int(sp[-1]):
        raise ValueError("seg_ids shorter than req_seg_ptr[-1]")
    h = _P()
    _check(load_library().tl_plan_create(C.byref(h), pool, q_heads, len(rp) - 1, _addr(rp), _addr(sp),
                                         _addr(ids) if len(ids) else None, flags, split_segments, compute_units))
    return h.value


def tl_plan_destroy(plan: int):
    _plan_sizes.pop(plan, None)
    _check(load_library().tl_plan_destroy(plan))


# What the tensors of a compute call need at least, for every live plan: elements of (q and the output, new K or V,
# the output's LSE, the partials, the partials' LSE).  The compute wrappers check the tensors they are handed
# against it -- the C ABI sees only pointers and cannot.
_plan_sizes = {}


def _sizes_of(plan: int):
    sz = _plan_sizes.get(plan)
    if sz is None:
        i = tl_plan_get_info(plan)
        T, R, hq, hkv = i.n_tokens, i.n_partial_rows, i.q_heads, i.kv_heads
        sz = _plan_sizes[plan] = (T * hq * 128, T * hkv * 128, T * hq, R * hq * 128, R * hq)
    return sz


def _need(t, name: str, n: int, kind: str) -> Optional[int]:
    """The address of t, a dense device tensor of the given element kind with at least n elements (or an address,
    or None); a tensor that the plan has no rows for may be anything dense."""
    if t is None or isinstance(t, int):
        return t
    if n:
        if not _kinds:
            import torch
            _kinds.update(bf16=torch.bfloat16, f32=torch.float32)
        if t.dtype != _kinds[kind]:
            raise TypeError("%s must be %s, is %s" % (name, kind, t.dtype))
        if t.numel() < n:
            raise ValueError("%s has %d elements, the plan needs %d" % (name, t.numel(), n))
    if not t.is_contiguous():
        raise ValueError("device tensor must be contiguous")
    return t.data_ptr()


_kinds = {}


def tl_plan_get_info(plan: int) -> tl_plan_info:
    info = tl_plan_info()
    _check(load_library().tl_plan_get_info(plan, C.byref(info)))
    return info


def tl_plan_hot_slots(plan: int, max_n: int):
    """(slots, loads) of the batch's most loaded slots, at most max_n."""
    slots, loads, n = np.zeros(max(max_n, 1), np.int32), np.zeros(max(max_n, 1), np.int64), _I32(0)
    _check(load_library().tl_plan_hot_slots(plan, max_n, slots.ctypes.data, loads.ctypes.data, C.byref(n)))
    return slots[:n.value], loads[:n.value]


def tl_plan_export(plan: int) -> dict:
    lib = load_library()
    info = tl_plan_get_info(plan)
    nt, ns = _I32(0), _I32(0)
    _check(lib.tl_plan_export_sizes(plan, C.byref(nt), C.byref(ns)))
    out = {
        "item_row_base": np.zeros(info.n_items, np.int32),
        "item_tok_ptr": np.zeros(info.n_items + 1, np.int32),
        "item_tokens": np.zeros(nt.value, np.int32),
        "item_slot_ptr": np.zeros(info.n_items + 1, np.int32),
        "item_slots": np.zeros(ns.value, np.int32),
        "merge_ptr": np.zeros(info.n_tokens + 1, np.int32),
        "merge_rows": np.zeros(info.n_merge_entries, np.int32),
    }
    _check(lib.tl_plan_export(plan, *[out[k].ctypes.data for k in (
        "item_row_base", "item_tok_ptr", "item_tokens", "item_slot_ptr", "item_slots", "merge_ptr", "merge_rows")]))
    return out


# ---- compute ----------------------------------------------------------------------------
def tl_segment_attn(pool: int, plan: int, q, scale: float, out_partial, lse, stream=None):
    n_q, _, _, n_part, n_plse = _sizes_of(plan)
    _check(load_library().tl_segment_attn(pool, plan, _need(q, "q", n_q, "bf16"), scale, _need(out_partial, "out_partial", n_part, "f32"),
                                          _need(lse, "lse", n_plse, "f32"), _stream(stream)))


def tl_causal_block(plan: int, q, k_new, v_new, scale: float, out_partial, lse, stream=None):
    n_q, n_kv, _, n_part, n_plse = _sizes_of(plan)
    _check(load_library().tl_causal_block(plan, _need(q, "q", n_q, "bf16"), _need(k_new, "k_new", n_kv, "bf16"),
                                          _need(v_new, "v_new", n_kv, "bf16"), scale, _need(out_partial, "out_partial", n_part, "f32"),
                                          _need(lse, "lse", n_plse, "f32"), _stream(stream)))


def _fused_args(pool, plan, q, k_new, v_new, scale, out, out_is_bf16, lse_out, stream, prior_partial, prior_lse):
    n_q, n_kv, n_lse, n_part, n_plse = _sizes_of(plan)
    return (pool, plan, _need(q, "q", n_q, "bf16"), _need(k_new, "k_new", n_kv, "bf16"), _need(v_new, "v_new", n_kv, "bf16"), scale,
            _need(prior_partial, "prior_partial", n_part, "f32"), _need(prior_lse, "prior_lse", n_plse, "f32"),
            _need(out, "out", n_q, "bf16" if out_is_bf16 else "f32"), int(bool(out_is_bf16)), _need(lse_out, "lse_out", n_lse, "f32"),
            _stream(stream))


def tl_fused_attn(pool: int, plan: int, q, k_new, v_new, scale: float, out, out_is_bf16: bool, lse_out=None, stream=None,
                  prior_partial=None, prior_lse=None):
    """prior_partial / prior_lse: the partial buffers tl_segment_attn wrote (needed by TL_PLAN_FUSE_TAILS plans)."""
    _check(load_library().tl_fused_attn(*_fused_args(pool, plan, q, k_new, v_new, scale, out, out_is_bf16, lse_out, stream,
                                                     prior_partial, prior_lse)))


def tl_fused_attn_static(pool: int, plan: int, q, k_new, v_new, scale: float, out, out_is_bf16: bool, lse_out=None,
                         stream=None, prior_partial=None, prior_lse=None):
    """tl_fused_attn without any device allocation (the plan's work lists go to a static device buffer)."""
    _check(load_library().tl_fused_attn_static(*_fused_args(pool, plan, q, k_new, v_new, scale, out, out_is_bf16, lse_out, stream,
                                                            prior_partial, prior_lse)))


def tl_merge(plan: int, out_partial, lse, out, out_is_bf16: bool, lse_out=None, stream=None):
    n_q, _, n_lse, n_part, n_plse = _sizes_of(plan)
    _check(load_library().tl_merge(plan, _need(out_partial, "out_partial", n_part, "f32"), _need(lse, "lse", n_plse, "f32"),
                                   _need(out, "out", n_q, "bf16" if out_is_bf16 else "f32"), int(bool(out_is_bf16)),
                                   _need(lse_out, "lse_out", n_lse, "f32"), _stream(stream)))


# ---- rows between the projection and the attention -----------------------------------------
def tl_rope_steps(inv_freq) -> np.ndarray:
    """uint64 [rot_dim / 2]; what tl_rope_of takes is `torch.from_numpy(steps.view(np.int64))` on the device."""
    f = _host(inv_freq, np.float64)
    steps = np.zeros(len(f), np.uint64)
    _check(load_library().tl_rope_steps(_addr(f) if len(f) else None, len(f), _addr(steps) if len(f) else None))
    return steps


def tl_rope_of(steps, interleaved: bool = False, factor: float = 1.0) -> tl_rope:
    """steps: int64 device tensor [rot_dim / 2] with the bits of tl_rope_steps; the struct keeps it alive."""
    device = max(steps.get_device(), 0)
    rope = tl_rope(_dense(steps, "steps", _row_kinds()["i64"], steps.numel(), device), 2 * steps.numel(), int(bool(interleaved)), factor)
    rope.steps, rope.device = steps, device
    return rope


_ROW_KINDS = {}
_MOST_ROWS = (1 << 31) - 1      # the C side counts in 32 bits, and ctypes would cut a larger number to them


def _row_kinds():
    if not _ROW_KINDS:
        import torch
        _ROW_KINDS.update(bf16=torch.bfloat16, f32=torch.float32, i32=torch.int32, i64=torch.int64,
                          current=getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device))
    return _ROW_KINDS


def _dense(t, name, kind, n, device):
    """Address of a dense device tensor of n elements."""
    if t.dtype is not kind:
        raise TypeError("%s must be %s, is %s" % (name, kind, t.dtype))
    if t.get_device() != device:
        raise ValueError("%s is on another device" % name)
    if t.numel() != n or not t.is_contiguous():
        raise ValueError("%s must be dense with %d elements, is %s with strides %s" % (name, n, tuple(t.shape), t.stride()))
    return t.data_ptr()


def _in_order(shape, n, heads):
    """Whether the elements of a dense tensor of this shape are those of [n, heads, 128] in that order: a flat one, leading dimensions of n tokens
    or of n heads of all tokens, values last.  ([heads, n, 128] would be filled with tokens and heads mixed up.)"""
    dims = [d for d in shape if d != 1]
    return math.prod(dims) == n * heads * 128 and (
        len(dims) < 2 or dims[-1] % 128 == 0 and (n == 1 or dims[0] == n * heads or n in accumulate(dims[:-1], mul)))


def _out_of(t, name, bf16, n, heads, device):
    """Address of a dense output [n, heads, 128], or of one of another shape with the same order."""
    if t.dtype is not bf16:
        raise TypeError("%s must be %s, is %s" % (name, bf16, t.dtype))
    if t.get_device() != device:
        raise ValueError("%s is on another device" % name)
    shape = t.shape
    if (shape != (n, heads, 128) and not _in_order(shape, n, heads)) or not t.is_contiguous():
        raise ValueError("%s must be dense [%d, %d, 128], is %s with strides %s" % (name, n, heads, tuple(shape), t.stride()))
    return t.data_ptr()


# tl_qkv as bytes: filling the ctypes structure field by field takes 0.8 us, this 0.2
_PACK_QKV = Struct("3Q6q3if5Q").pack


def _rows_of(x, name, dtype, device):
    """(address, tokens, heads, stride between tokens, between heads) of [n, heads, 128]; the values of a head follow each other."""
    if x.dtype is not dtype:
        raise TypeError("%s must be %s, is %s" % (name, dtype, x.dtype))
    if x.get_device() != device:
        raise ValueError("%s is on another device" % name)
    shape, stride = x.shape, x.stride()
    if len(shape) != 3 or shape[2] != 128 or stride[2] != 1:
        raise ValueError("%s must be [n, heads, 128] with adjacent values, is %s with strides %s" % (name, tuple(shape), stride))
    return x.data_ptr(), shape[0], shape[1], stride[0], stride[1]


def _qkv(rope, pos, q, k, v, q_out, k_out, v_out, q_weight, k_weight, eps):
    """(tl_qkv's bytes, positions, tokens, device) of a call: shapes, types, strides and devices of its tensors are checked here."""
    # (a decoded token's call takes as long here as in the launch: tensors are asked for what is looked at, once)
    kinds = _ROW_KINDS or _row_kinds()
    some = q if q is not None else k if k is not None else v
    if some is None:
        raise ValueError("no rows")
    dtype, device, bf16, f32 = some.dtype, some.get_device(), kinds["bf16"], kinds["f32"]
    if device < 0 or device != kinds["current"]():
        raise ValueError("rows must be on the current device")
    if dtype is not bf16 and dtype is not f32:
        raise TypeError("rows must be bf16 or f32, are %s" % dtype)
    qp = kp = vp = qn = kn = vn = qh = kh = vh = qr = qs = kr = ks = vr = vs = qo = ko = vo = qw = kw = 0
    if q is not None:
        qp, qn, qh, qr, qs = _rows_of(q, "q", dtype, device)
    if k is not None:
        kp, kn, kh, kr, ks = _rows_of(k, "k", dtype, device)
    if v is not None:
        vp, vn, vh, vr, vs = _rows_of(v, "v", dtype, device)
    n = qn or kn or vn
    if (q is not None and qn != n) or (k is not None and kn != n) or (v is not None and vn != n) or (k is not None and v is not None and kh != vh):
        raise ValueError("q, k and v of %d, %d and %d tokens, k and v of %d and %d heads" % (qn, kn, vn, kh, vh))
    if n > _MOST_ROWS:
        raise ValueError("%d tokens in one call" % n)
    if q_out is not None:
        qo = _out_of(q_out, "q_out", bf16, n, qh, device)
    if k_out is not None:
        ko = _out_of(k_out, "k_out", bf16, n, kh, device)
    if v_out is not None:
        vo = _out_of(v_out, "v_out", bf16, n, vh, device)
    if q_weight is not None:
        qw = _dense(q_weight, "q_weight", f32, 128, device)
    if k_weight is not None:
        kw = _dense(k_weight, "k_weight", f32, 128, device)
    at = None
    if rope is not None:
        if rope.device != device:
            raise ValueError("the rotation's steps are on another device")
        if pos is not None:
            at = _dense(pos, "pos", kinds["i32"], n, device)
    return _PACK_QKV(qp, kp, vp, qr, qs, kr, ks, vr, vs, qh, kh or vh, dtype is bf16, eps, qw, kw, qo, ko, vo), at, n, device


def _at(rope) -> Optional[int]:
    return None if rope is None else C.addressof(rope)


def tl_rotate_rows(rope: Optional[tl_rope], pos, q=None, k=None, v=None, q_out=None, k_out=None, v_out=None, q_weight=None, k_weight=None,
                   eps: float = 1e-6, stream=None):
    """Norms (with weights) and rotation (with rope) of q [n, q_heads, 128] and k [n, kv_heads, 128] with any strides between tokens and
    heads, bf16 or fp32; v as it is; to dense bf16 tensors [n, heads, 128] (of any shape with that order: [n, heads * 128], [batch, length, heads, 128]).
    pos: int32, n of them."""
    rows, at, n, _ = _qkv(rope, pos, q, k, v, q_out, k_out, v_out, q_weight, k_weight, eps)
    _check(load_library().tl_rotate_rows(_at(rope), rows, at, n, _stream(stream)))


def tl_pool_write_rows(pool: int, rope: Optional[tl_rope], pos, pool_rows, k, v, q=None, q_out=None, k_out=None, v_out=None, q_weight=None,
                       k_weight=None, eps: float = 1e-6, stream=None):
    """tl_rotate_rows that writes k and v to the pool: token i's to pool row pool_rows[i] (int32, n of them; -1: nowhere)."""
    rows, at, n, device = _qkv(rope, pos, q, k, v, q_out, k_out, v_out, q_weight, k_weight, eps)
    _check(load_library().tl_pool_write_rows(pool, _at(rope), rows, at, _dense(pool_rows, "pool_rows", _ROW_KINDS["i32"], n, device), n,
                                             _stream(stream)))


def tl_pool_move_rows(pool: int, rope: Optional[tl_rope], src_rows, dst_rows, shift=None, stream=None):
    """Pool row src_rows[i] to dst_rows[i], keys turned on by shift[i] positions (int32, as many of each)."""
    kinds = _ROW_KINDS or _row_kinds()
    i32, n, device = kinds["i32"], src_rows.numel(), src_rows.get_device()
    if device < 0 or device != kinds["current"]():
        raise ValueError("rows must be on the current device")
    if n > _MOST_ROWS:
        raise ValueError("%d rows in one call" % n)
    src, dst = _dense(src_rows, "src_rows", i32, n, device), _dense(dst_rows, "dst_rows", i32, n, device)
    at = None
    if rope is not None:
        if rope.device != device:
            raise ValueError("the rotation's steps are on another device")
        if shift is not None:
            at = _dense(shift, "shift", i32, n, device)
    _check(load_library().tl_pool_move_rows(pool, _at(rope), src, dst, at, n, _stream(stream)))


def tl_set_option(knob: str, value: int):
    _check(load_library().tl_set_option(knob.encode(), value))


# ---- analytic models ----------------------------------------------------------------------
def tl_model_segment_time(n_tokens: float, d_q: float, d_kv: float, flops: float, mem_bw: float) -> float:
    out = _F64(0.0)
    _check(load_library().tl_model_segment_time(n_tokens, d_q, d_kv, flops, mem_bw, C.byref(out)))
    return out.value


def tl_model_comm_time(d_q: float, net_latency: float, net_bw: float) -> float:
    out = _F64(0.0)
    _check(load_library().tl_model_comm_time(d_q, net_latency, net_bw, C.byref(out)))
    return out.value


def tl_model_segment_threshold(d_q: float, d_kv: float, flops: float, mem_bw: float, net_latency: float,
                               net_bw: float) -> float:
    out = _F64(0.0)
    _check(load_library().tl_model_segment_threshold(d_q, d_kv, flops, mem_bw, net_latency, net_bw, C.byref(out)))
    return out.value


def tl_model_cache_load(d: float, prefix_len, input_len, n_gpus: int, mem_bw: float, flops: float, t_ideal: float):
    """Returns (M_r bytes, F_r flop, L)."""
    pl, il = _host(prefix_len, np.int64), _host(input_len, np.int64)
    if len(pl) != len(il):
        raise ValueError("prefix_len/input_len length mismatch")
    m, f, load = _F64(0.0), _F64(0.0), _F64(0.0)
    _check(load_library().tl_model_cache_load(d, pl.ctypes.data if len(pl) else None, il.ctypes.data if len(il) else None,
                                              len(pl), n_gpus, mem_bw, flops, t_ideal, C.byref(m), C.byref(f), C.byref(load)))
    return m.value, f.value, load.value


def tl_segment_ids(tokens, seg_len: int, salt: int = 0) -> np.ndarray:
    """Content-derived ids of the segments of a token sequence (uint64, one per started segment)."""
    t = _host(tokens, np.int32)
    n_ids = (len(t) + seg_len - 1) // seg_len if seg_len > 0 else 0
    ids = np.zeros(n_ids, np.uint64)
    _check(load_library().tl_segment_ids(t.ctypes.data if len(t) else None, len(t), seg_len, salt & 0xFFFFFFFFFFFFFFFF,
                                         ids.ctypes.data if n_ids else None))
    return ids
