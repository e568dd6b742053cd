"""Binding of liblserve.so: argument marshalling only, every step runs in the HIP kernels.  The calls of a decode step and
those on new tokens are marshalled natively (csrc/py_calls.cpp), the others by ctypes."""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import warnings
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# LSERVE_LIBRARY points at another build of the same library (e.g. an instrumented one)
_LIB_PATH = os.environ.get("LSERVE_LIBRARY") or os.path.join(_HERE, "liblserve.so")
_lib = None
_calls = None

LSERVE_CALL_BUILD_PAGE_STATS = 0
LSERVE_CALL_SELECT_PAGES = 1
LSERVE_CALL_SPARSE_PREFILL = 2
LSERVE_CALL_SPARSE_DECODE = 3
LSERVE_TREE_WORKSPACE_MOST = 352 << 20

EXPORTED_SYMBOLS = (
    "lserve_build_page_stats",
    "lserve_select_pages",
    "lserve_sparse_prefill",
    "lserve_sparse_decode",
    "lserve_append_kv",
    "lserve_sparse_prefill_masked",
    "lserve_sparse_prefill_paged",
    "lserve_sparse_prefill_chunk",
    "lserve_chunk_scratch_bytes",
    "lserve_paged_prefill_workspace_bytes",
    "lserve_masked_prefill_workspace_bytes",
    "BlockMask",
    "lserve_workspace_bytes",
    "lserve_strerror",
    "lserve_last_hip_error",
    "lserve_init",
    "lserve_sparse_decode_noalloc",
    "lserve_probe_decode_read",
    "lserve_probe_prefill_shape",
    "lserve_probe_prefill_plan",
    "lserve_probe_prefill_longest_first",
    "lserve_probe_mask_walk",
    "lserve_extend_tables",
    "lserve_rotary",
    "lserve_rotary_frequencies",
    "RotaryDesc",
    "lserve_rotary_axes",
    "PositionAxes",
    "lserve_norm_rotary",
    "HeadNorm",
    "lserve_rotary_append_kv",
    "lserve_tree_masks",
    "lserve_sparse_decode_tree",
    "lserve_tree_workspace_bytes",
)


class LserveError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where} failed with code {code}: {lserve_strerror(code)}"
                         + (f" (hipError_t {lserve_last_hip_error()})" if code == -4 else ""))


class _CAttnDesc(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int32), ("num_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
        ("page_size", ctypes.c_int32), ("logical_page_size", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("sink_tokens", ctypes.c_int32), ("local_tokens", ctypes.c_int32),
        ("kv_head_is_streaming", ctypes.POINTER(ctypes.c_uint8)), ("sm_scale", ctypes.c_float),
    ]


class _CPagedKV(ctypes.Structure):
    _fields_ = [
        ("k_pool", ctypes.c_void_p), ("v_pool", ctypes.c_void_p), ("stats", ctypes.c_void_p),
        ("page_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
        ("batch", ctypes.c_int32), ("max_pages_per_seq", ctypes.c_int32), ("num_pages", ctypes.c_int32),
        ("pool_heads", ctypes.c_int32),
        ("k_pool_stream", ctypes.c_void_p), ("v_pool_stream", ctypes.c_void_p), ("ring_table", ctypes.c_void_p),
        ("num_pages_stream", ctypes.c_int32), ("kv_bits", ctypes.c_int32),
    ]


class _CBlockMask(ctypes.Structure):
    _fields_ = [
        ("head_mask", ctypes.c_void_p), ("q_tile_start", ctypes.c_void_p), ("row_ptr", ctypes.c_void_p),
        ("cols", ctypes.c_void_p),
        ("num_masks", ctypes.c_int32), ("rows_per_mask", ctypes.c_int32), ("nnz", ctypes.c_int32),
    ]


class _CRotaryDesc(ctypes.Structure):
    _fields_ = [("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("inv_freq", ctypes.c_void_p), ("scale", ctypes.c_float)]


class _CPositionAxes(ctypes.Structure):
    _fields_ = [("num_axes", ctypes.c_int32), ("pair_axis", ctypes.POINTER(ctypes.c_uint8))]


class _CHeadNorm(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("per_head", ctypes.c_int32), ("eps", ctypes.c_float), ("q_weight", ctypes.c_void_p),
                ("k_weight", ctypes.c_void_p)]


class _CRotaryScaling(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("rotary_dim", ctypes.c_int32), ("base", ctypes.c_double), ("factor", ctypes.c_double),
                ("original_positions", ctypes.c_double), ("low", ctypes.c_double), ("high", ctypes.c_double)]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load liblserve.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise FileNotFoundError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2502_14866_amd.build` "
                "(or __graft_entry__.build()); there is no CPU fallback")
        lib = ctypes.CDLL(_LIB_PATH)
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        dp, kp = ctypes.POINTER(_CAttnDesc), ctypes.POINTER(_CPagedKV)
        lib.lserve_build_page_stats.argtypes = [dp, kp, vp, i32, vp]
        lib.lserve_select_pages.argtypes = [dp, kp, vp, i32, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.lserve_sparse_prefill.argtypes = [dp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_decode.argtypes = [dp, kp, vp, vp, vp, vp, i32, vp, vp, vp, sz, vp]
        lib.lserve_append_kv.argtypes = [dp, kp, vp, vp, vp, vp, i32, vp]
        lib.lserve_append_kv.restype = ctypes.c_int
        mp = ctypes.POINTER(_CBlockMask)
        lib.lserve_sparse_prefill_masked.argtypes = [dp, mp, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_prefill_masked.restype = ctypes.c_int
        lib.lserve_masked_prefill_workspace_bytes.argtypes = [dp, i32, i32, i32, i32, i32]
        lib.lserve_masked_prefill_workspace_bytes.restype = ctypes.c_size_t
        lib.lserve_sparse_prefill_paged.argtypes = [dp, kp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_prefill_paged.restype = ctypes.c_int
        lib.lserve_sparse_prefill_paged_scratch.argtypes = [dp, kp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_prefill_paged_scratch.restype = ctypes.c_int
        lib.lserve_sparse_prefill_chunk.argtypes = [dp, kp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
        lib.lserve_sparse_prefill_chunk.restype = ctypes.c_int
        lib.lserve_sparse_prefill_chunk_scratch.argtypes = [dp, kp, vp, vp, vp, vp, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_prefill_chunk_scratch.restype = ctypes.c_int
        lib.lserve_chunk_scratch_bytes.argtypes = [dp, i32, i32, i32, i32, i32]
        lib.lserve_chunk_scratch_bytes.restype = sz
        lib.lserve_paged_prefill_workspace_bytes.argtypes = [dp, i32, i32]
        lib.lserve_paged_prefill_workspace_bytes.restype = ctypes.c_size_t
        lib.lserve_workspace_bytes.argtypes = [ctypes.c_int, dp, i32, i32, i32, i32]
        lib.lserve_workspace_bytes.restype = sz
        lib.lserve_strerror.argtypes = [ctypes.c_int]
        lib.lserve_strerror.restype = ctypes.c_char_p
        lib.lserve_last_hip_error.restype = ctypes.c_int
        lib.lserve_sparse_decode_noalloc.argtypes = [dp, kp, vp, vp, vp, vp, i32, vp, vp, vp]
        lib.lserve_sparse_decode_noalloc.restype = ctypes.c_int
        lib.lserve_probe_decode_read.argtypes = [dp, kp, vp, vp, vp, i32, vp]
        lib.lserve_probe_decode_read.restype = ctypes.c_int
        lib.lserve_probe_prefill_shape.argtypes = [dp, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
        lib.lserve_probe_prefill_shape.restype = ctypes.c_int
        lib.lserve_probe_prefill_plan.argtypes = [dp, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
        lib.lserve_probe_prefill_plan.restype = ctypes.c_int
        lib.lserve_probe_prefill_longest_first.argtypes = [dp, i32, i32, i32, ctypes.POINTER(i32)]
        lib.lserve_probe_prefill_longest_first.restype = ctypes.c_int
        lib.lserve_probe_mask_walk.argtypes = [dp, i32, i32, i32, i32, i32, i32, ctypes.POINTER(i32)]
        lib.lserve_probe_mask_walk.restype = ctypes.c_int
        lib.lserve_extend_tables.argtypes = [dp, kp, vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp]
        lib.lserve_extend_tables.restype = ctypes.c_int
        i64 = ctypes.c_int64
        lib.lserve_rotary.argtypes = [dp, ctypes.POINTER(_CRotaryDesc), vp, vp, vp, i32, i64, i64, vp, vp, vp]
        lib.lserve_rotary.restype = ctypes.c_int
        lib.lserve_rotary_frequencies.argtypes = [ctypes.POINTER(_CRotaryScaling), vp, vp]
        lib.lserve_rotary_frequencies.restype = ctypes.c_int
        rp, ap, np_ = ctypes.POINTER(_CRotaryDesc), ctypes.POINTER(_CPositionAxes), ctypes.POINTER(_CHeadNorm)
        lib.lserve_rotary_axes.argtypes = [dp, rp, ap, vp, vp, vp, i64, i32, i64, i64, vp, vp, vp]
        lib.lserve_rotary_axes.restype = ctypes.c_int
        lib.lserve_norm_rotary.argtypes = [dp, np_, rp, ap, vp, vp, vp, i64, i32, i64, i64, vp, vp, vp]
        lib.lserve_norm_rotary.restype = ctypes.c_int
        lib.lserve_rotary_append_kv.argtypes = [dp, kp, np_, rp, ap, vp, vp, vp, i64, i64, i64, vp, i64, vp, vp, i32, i32, vp, vp, vp, vp]
        lib.lserve_rotary_append_kv.restype = ctypes.c_int
        lib.lserve_tree_masks.argtypes = [vp, vp, vp, i32, i32, i32, i32, vp, vp, vp]
        lib.lserve_tree_masks.restype = ctypes.c_int
        lib.lserve_sparse_decode_tree.argtypes = [dp, kp, vp, vp, vp, vp, vp, i32, vp, vp, vp, vp, i32, i32, i32, vp, vp, vp, sz, vp]
        lib.lserve_sparse_decode_tree.restype = ctypes.c_int
        lib.lserve_tree_workspace_bytes.argtypes = [dp, i32, i32, i32, i32, i32]
        lib.lserve_tree_workspace_bytes.restype = sz
        lib.lserve_init.argtypes = []
        lib.lserve_init.restype = ctypes.c_int
        for name in ("lserve_build_page_stats", "lserve_select_pages", "lserve_sparse_prefill",
                     "lserve_sparse_decode"):
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


class _CtypesCalls:
    """The native calls by ctypes, where the extension is not there or not of this torch; desc as its address."""

    @staticmethod
    def append(desc, kv, k_new, v_new, cu_new, start_pos, max_new_per_seq, stream):
        return load_library().lserve_append_kv(_CAttnDesc.from_address(desc), kv.c(), _ptr(k_new), _ptr(v_new), _ptr(cu_new),
                                               _ptr(start_pos), max_new_per_seq, stream)

    @staticmethod
    def select(desc, kv, q, budget_tokens, stats_valid_len, sel_pages, sel_count, sel_seq_len, scores_out, workspace, stream):
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        return load_library().lserve_select_pages(_CAttnDesc.from_address(desc), kv.c(), _ptr(q), budget_tokens,
                                                  _ptr(stats_valid_len), _ptr(sel_pages), _ptr(sel_count), _ptr(sel_seq_len),
                                                  _ptr(scores_out), _ptr(workspace), ws_bytes, stream)

    @staticmethod
    def decode(desc, kv, q, sel_pages, sel_count, sel_seq_len, out, lse_out, workspace, stream):
        ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
        sel_stride = 0 if sel_pages is None else sel_pages.shape[-1]
        return load_library().lserve_sparse_decode(_CAttnDesc.from_address(desc), kv.c(), _ptr(q), _ptr(sel_pages),
                                                   _ptr(sel_count), _ptr(sel_seq_len), sel_stride, _ptr(out), _ptr(lse_out),
                                                   _ptr(workspace), ws_bytes, stream)


    @staticmethod
    def extend(desc, kv, new_lens, free_pages, cu_new, new_seq_lens, pages_taken, positions, slots, ring_slots, total_new, stream):
        d, batch, i32, i64 = _CAttnDesc.from_address(desc), kv.page_table.shape[0], torch.int32, torch.int64
        _checked("lserve_extend_tables", (kv.page_table, i32, 0), (kv.seq_lens, i32, batch), (kv.ring_table, i32, 0), (new_lens, i32, batch),
                 (free_pages, i32, 0), (cu_new, i32, batch + 1), (new_seq_lens, i32, batch), (pages_taken, i32, 1),
                 (positions, i32, total_new), (slots, i64, total_new), (ring_slots, i64, total_new))
        if ring_slots is not None and kv.ring_table is not None and kv.ring_table.numel() < batch * _ring(d):
            raise ValueError(f"lserve_extend_tables: a ring table of {kv.ring_table.numel()} entries for {batch} sequences of {_ring(d)}")
        return load_library().lserve_extend_tables(
            d, kv.c(), _ptr(new_lens), _ptr(free_pages), 0 if free_pages is None else free_pages.numel(), total_new, _ptr(cu_new),
            _ptr(new_seq_lens), _ptr(pages_taken), _ptr(positions), _ptr(slots), _ptr(ring_slots), stream)

    @staticmethod
    def masks(parents, cu_new, seq_lens, max_new_per_seq, tree_mask, positions, stream):
        total, batch = (0 if parents is None else parents.numel()), (0 if cu_new is None else cu_new.numel() - 1)
        words = 0 if tree_mask is None else tree_mask.shape[-1]
        _checked("lserve_tree_masks", (parents, torch.int32, 1), (cu_new, torch.int32, 2), (seq_lens, torch.int32, batch),
                 (tree_mask, torch.int64, total * words), (positions, torch.int32, total))
        return load_library().lserve_tree_masks(_ptr(parents), _ptr(cu_new), _ptr(seq_lens), batch, total, max_new_per_seq, words,
                                                _ptr(tree_mask), _ptr(positions), stream)

    @staticmethod
    def rotary(desc, rotary, inv_freq, q, k, positions, q_out, k_out, stream):
        d, r = _CAttnDesc.from_address(desc), _CRotaryDesc.from_address(rotary)
        total, dim, hq, hkv, dt = (0 if positions is None else positions.numel()), d.head_dim, d.num_q_heads, d.num_kv_heads, _dtype(d)
        (q_at, q_stride), (k_at, k_stride) = _rows("lserve_rotary", q, hq, dim, "q"), _rows("lserve_rotary", k, hkv, dim, "k")
        _checked("lserve_rotary", (positions, torch.int32, 1), (inv_freq, torch.float64, r.rotary_dim // 2 if r.rotary_dim <= dim else 0), (q, dt, total * hq * dim),
                 (q_out, dt, total * hq * dim), (k, dt, total * hkv * dim), (k_out, dt, total * hkv * dim))
        return load_library().lserve_rotary(d, _rotary_struct(rotary, inv_freq), q_at, k_at, _ptr(positions), total, q_stride, k_stride, _ptr(q_out), _ptr(k_out), stream)

    @staticmethod
    def turned(desc, norm, rotary, axes, q_weight, k_weight, inv_freq, q, k, positions, q_out, k_out, stream):
        where = "lserve_norm_rotary" if norm else "lserve_rotary_axes"
        d, dt = _CAttnDesc.from_address(desc), _dtype(_CAttnDesc.from_address(desc))
        dim, hq, hkv = d.head_dim, d.num_q_heads, d.num_kv_heads
        total = positions.shape[-1] if positions is not None and positions.dim() else q.shape[0] if q is not None else 0 if k is None else k.shape[0]
        (q_at, q_stride), (k_at, k_stride) = _rows(where, q, hq, dim, "q"), _rows(where, k, hkv, dim, "k")
        at, apart = _places(where, positions, axes, total)
        _checked(where, *_turn_tensors(d, norm, rotary, q_weight, k_weight, inv_freq), (positions, torch.int32, 1), (q, dt, total * hq * dim),
                 (q_out, dt, total * hq * dim), (k, dt, total * hkv * dim), (k_out, dt, total * hkv * dim))
        lib, n, r, a = load_library(), _norm_struct(norm, q_weight, k_weight), _rotary_struct(rotary, inv_freq), _struct(_CPositionAxes, axes)
        if norm:
            return lib.lserve_norm_rotary(d, n, r, a, q_at, k_at, at, apart, total, q_stride, k_stride, _ptr(q_out), _ptr(k_out), stream)
        return lib.lserve_rotary_axes(d, r, a, q_at, k_at, at, apart, total, q_stride, k_stride, _ptr(q_out), _ptr(k_out), stream)

    @staticmethod
    def rotary_append(desc, kv, norm, rotary, axes, q_weight, k_weight, inv_freq, q, k, v, positions, cu_new, start_pos, max_new_per_seq, q_out, k_out,
                      v_out, stream):
        where, d, i32 = "lserve_rotary_append_kv", _CAttnDesc.from_address(desc), torch.int32
        dt, dim, hq, hkv, batch = _dtype(d), d.head_dim, d.num_q_heads, d.num_kv_heads, kv.page_table.shape[0]
        total = 0 if k is None or not k.dim() else k.shape[0]
        rows = [_rows(where, t, heads, dim, name) for t, heads, name in ((q, hq, "q"), (k, hkv, "k"), (v, hkv, "v"))]
        at, apart = _places(where, positions, axes, total)
        kind, slab = _slab(d, kv.kv_bits)
        streaming = sum(1 for f in d.kv_head_is_streaming[:hkv] if f)
        streams = streaming if kv.k_pool_stream is not None else 0
        kv.c()
        heads = kv._c.num_pages * (kv.pool_heads or hkv) if streams < hkv else 0  # (all heads in the bounded pool: nothing of the main one)
        spans = heads * (d.page_size // d.logical_page_size if d.logical_page_size > 0 else 0) * 2 * dim if streaming < hkv else 0
        pool, bounded = heads * slab, kv._c.num_pages_stream * streams * slab
        _checked(where, *_turn_tensors(d, norm, rotary, q_weight, k_weight, inv_freq), (q, dt, total * hq * dim), (k, dt, total * hkv * dim),
                 (v, dt, total * hkv * dim), (positions, i32, 1), (cu_new, i32, batch + 1), (start_pos, i32, batch), (q_out, dt, total * hq * dim),
                 (k_out, dt, total * hkv * dim), (v_out, dt, total * hkv * dim), (kv.page_table, i32, 0), (kv.k_pool, kind, pool),
                 (kv.v_pool, kind, pool), (kv.k_pool_stream, kind, bounded), (kv.v_pool_stream, kind, bounded), (kv.stats, dt, spans),
                 (kv.ring_table, i32, batch * _ring(d) if kv.k_pool_stream is not None else 0))
        return load_library().lserve_rotary_append_kv(
            d, kv.c(), _norm_struct(norm, q_weight, k_weight), _rotary_struct(rotary, inv_freq), _struct(_CPositionAxes, axes), rows[0][0], rows[1][0], rows[2][0],
            rows[0][1], rows[1][1], rows[2][1], at, apart, _ptr(cu_new), _ptr(start_pos), total, max_new_per_seq, _ptr(q_out), _ptr(k_out), _ptr(v_out),
            stream)

    @staticmethod
    def tree(desc, kv, q, k_new, v_new, cu_new, max_new_per_seq, out, lse_out, tree_mask, positions, sel_pages, sel_count, sel_seq_len,
             workspace, stream):
        d, batch, i32 = _CAttnDesc.from_address(desc), kv.page_table.shape[0], torch.int32
        total, dim, hq, hkv, dt = (0 if q is None else q.shape[0]), d.head_dim, d.num_q_heads, d.num_kv_heads, _dtype(d)
        words = 0 if tree_mask is None else tree_mask.shape[-1]
        stride = 0 if sel_pages is None else sel_pages.shape[-1]
        kind, slab = _slab(d, kv.kv_bits)
        streams = sum(d.kv_head_is_streaming[:hkv]) if kv.k_pool_stream is not None else 0
        kv.c()
        # (a layer whose heads are all in the bounded pool reads nothing of the main one)
        pool, bounded = kv._c.num_pages * (kv.pool_heads or hkv) * slab if streams < hkv else 0, kv._c.num_pages_stream * streams * slab
        _checked("lserve_sparse_decode_tree", (q, dt, total * hq * dim), (k_new, dt, total * hkv * dim), (v_new, dt, total * hkv * dim),
                 (out, dt, total * hq * dim), (lse_out, torch.float32, total * hq), (cu_new, i32, batch + 1), (kv.seq_lens, i32, batch),
                 (kv.page_table, i32, 0), (kv.k_pool, kind, pool), (kv.v_pool, kind, pool), (kv.k_pool_stream, kind, bounded),
                 (kv.v_pool_stream, kind, bounded), (kv.ring_table, i32, batch * _ring(d) if kv.k_pool_stream is not None else 0),
                 (tree_mask, torch.int64, total * words), (positions, i32, total),
                 (sel_pages, i32, batch * hkv * stride), (sel_count, i32, batch * hkv), (sel_seq_len, i32, batch),
                 (workspace, () if workspace is None else workspace.dtype, 0))
        return load_library().lserve_sparse_decode_tree(
            d, kv.c(), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(cu_new), _ptr(tree_mask), words, _ptr(positions), _ptr(sel_pages),
            _ptr(sel_count), _ptr(sel_seq_len), stride, total, max_new_per_seq, _ptr(out), _ptr(lse_out), _ptr(workspace),
            0 if workspace is None else workspace.numel() * workspace.element_size(), stream)


def _dtype(desc: "_CAttnDesc") -> torch.dtype:
    return torch.bfloat16 if desc.dtype == 1 else torch.float16


def _ring(desc: "_CAttnDesc") -> int:
    """Entries of a sequence in the ring table of the two-way cache."""
    return -(-desc.sink_tokens // desc.page_size) - (-desc.local_tokens // desc.page_size) if desc.page_size > 0 else 0


def _slab(desc: "_CAttnDesc", bits: int) -> tuple:
    """(type, elements) of one head's rows in a page; with a number of bits that the library refuses, any type and none."""
    if bits in (0, 16):
        return _dtype(desc), max(0, desc.page_size * desc.head_dim)
    return (torch.uint8, 8 * desc.head_dim * bits + 256) if bits in (8, 4) else ((_dtype(desc), torch.uint8), 0)


def _checked(where: str, *args) -> None:
    """(tensor or None, type or types, least number of elements) each: what the library cannot see from an address."""
    device = None
    for t, kinds, least in args:
        if t is None:
            continue
        if t.dtype not in (kinds if isinstance(kinds, tuple) else (kinds,)):
            raise ValueError(f"{where}: a tensor of {t.dtype} where {kinds} is taken")
        if t.numel() < least:
            raise ValueError(f"{where}: a tensor of {t.numel()} elements where {least} are read or written")
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError(f"{where}: tensors on {device} and {t.device}")
    if device is not None and device.type == "cuda" and device.index != torch.cuda.current_device():
        raise ValueError(f"{where}: tensors on {device} while device {torch.cuda.current_device()} is current")


def _struct(kind, address: int):
    return kind.from_address(address) if address else None


def _rotary_struct(address: int, inv_freq: Optional[torch.Tensor]) -> Optional["_CRotaryDesc"]:
    """A description of rotary positions with its frequencies where they are now."""
    if not address:
        return None
    r = _CRotaryDesc.from_buffer_copy(_CRotaryDesc.from_address(address))
    r.inv_freq = _ptr(inv_freq) if r.inv_freq else None
    return r


def _norm_struct(address: int, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor]) -> Optional["_CHeadNorm"]:
    """A norm's description with its weights where they are now."""
    if not address:
        return None
    n = _CHeadNorm.from_buffer_copy(_CHeadNorm.from_address(address))
    n.q_weight, n.k_weight = _ptr(q_weight) if n.q_weight else None, _ptr(k_weight) if n.k_weight else None
    return n


def _turn_tensors(d: "_CAttnDesc", norm: int, rotary: int, q_weight, k_weight, inv_freq) -> tuple:
    """What describes how heads are normed and turned, for _checked."""
    dim, per_head = d.head_dim, bool(norm) and _CHeadNorm.from_address(norm).per_head
    turning = _CRotaryDesc.from_address(rotary).rotary_dim if rotary else 0
    return ((q_weight, torch.float32, dim * d.num_q_heads if per_head else dim), (k_weight, torch.float32, dim * d.num_kv_heads if per_head else dim),
            (inv_freq, torch.float64, turning // 2 if turning <= dim else 0))


def _places(where: str, positions: Optional[torch.Tensor], axes: int, total: int) -> tuple:
    """(address, elements between two axes) of positions [total], or with axes [axes][total], whose axes may lie apart."""
    if positions is None:
        return None, 0
    if not axes:
        if positions.dim() != 1 or positions.shape[0] < total:
            raise ValueError(f"{where}: positions are [total] without axes")
        return _ptr(positions), 0
    n = _CPositionAxes.from_address(axes).num_axes
    if positions.dim() != 2 or positions.shape[0] != n or positions.shape[1] < total or (positions.shape[1] > 1 and positions.stride(1) != 1):
        raise ValueError(f"{where}: positions are [{n}][total], those of an axis next to each other")
    return positions.data_ptr(), positions.stride(0) if n > 1 else positions.shape[1]


def _rows(where: str, t: Optional[torch.Tensor], heads: int, dim: int, what: str) -> tuple:
    """(address, elements between two rows) of [total][heads][dim] whose rows may lie apart."""
    if t is None:
        return None, 0
    if t.dim() != 3 or t.shape[1:] != (heads, dim) or t.stride(2) != 1 or t.stride(1) != dim:
        raise ValueError(f"{where}: {what} is [total][{heads}][{dim}], heads next to each other")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else heads * dim


def _native():
    """The native calls, bound to the loaded library; without the extension (only the library was built, or it was built with another
    torch or Python) the same by ctypes, some five microseconds a call slower."""
    global _calls
    if _calls is None:
        lib = load_library()
        try:
            from . import _calls as calls

            if calls.torch_version != torch.__version__:
                raise ImportError(f"_calls was built with torch {calls.torch_version}, this is {torch.__version__}")
            calls.bind(*(ctypes.cast(f, ctypes.c_void_p).value
                         for f in (lib.lserve_append_kv, lib.lserve_select_pages, lib.lserve_sparse_decode)))
            if hasattr(lib, "lserve_extend_tables"):  # what stands in for the library may have the decode step's calls alone
                calls.bind_new(*(ctypes.cast(f, ctypes.c_void_p).value
                                 for f in (lib.lserve_extend_tables, lib.lserve_tree_masks, lib.lserve_rotary, lib.lserve_sparse_decode_tree)))
            if hasattr(lib, "lserve_rotary_append_kv"):
                calls.bind_turned(*(ctypes.cast(f, ctypes.c_void_p).value
                                    for f in (lib.lserve_rotary_axes, lib.lserve_norm_rotary, lib.lserve_rotary_append_kv)))
        except ImportError as e:
            warnings.warn(f"the binding's native calls are missing ({e}): decode steps are marshalled by ctypes; build them with "
                          "`python -m paper_2502_14866_amd.build` (or __graft_entry__.build())", RuntimeWarning, stacklevel=3)
            calls = _CtypesCalls
        _calls = calls
    return _calls


@dataclass
class AttnDesc:
    """Mirror of lserve_attn_desc."""
    num_q_heads: int
    num_kv_heads: int
    streaming_flags: Sequence[int]
    head_dim: int = 128
    page_size: int = 64
    logical_page_size: int = 16
    dtype: torch.dtype = torch.float16
    sink_tokens: int = 128
    local_tokens: int = 512
    sm_scale: float = 0.0

    def __post_init__(self):
        flags = [1 if f else 0 for f in self.streaming_flags]
        self._flags = (ctypes.c_uint8 * max(1, len(flags)))(*flags)
        self._c = _CAttnDesc(
            self.num_q_heads, self.num_kv_heads, self.head_dim, self.page_size, self.logical_page_size,
            {torch.float16: 0, torch.bfloat16: 1}.get(self.dtype, -1), self.sink_tokens, self.local_tokens,
            ctypes.cast(self._flags, ctypes.POINTER(ctypes.c_uint8)), float(self.sm_scale))

        self._address = ctypes.addressof(self._c)

    def c(self):
        return ctypes.byref(self._c)


@dataclass
class PagedKV:
    """Mirror of lserve_paged_kv; keeps the tensors alive."""
    k_pool: Optional[torch.Tensor]
    v_pool: Optional[torch.Tensor]
    stats: Optional[torch.Tensor]
    page_table: torch.Tensor
    seq_lens: torch.Tensor
    # two-way cache: heads per page of the main pool (0 = all KV heads) and the streaming heads' bounded pool
    pool_heads: int = 0
    k_pool_stream: Optional[torch.Tensor] = None
    v_pool_stream: Optional[torch.Tensor] = None
    ring_table: Optional[torch.Tensor] = None
    # 16: pools of the layer's 16-bit dtype [pages, heads, N_P, D]; 8 or 4: quantised pages, uint8
    # [pages, heads, 64 * D * kv_bits / 8 + 256]
    kv_bits: int = 16

    def c(self):
        sized = self.stats if self.stats is not None else self.v_pool if self.v_pool is not None else self.k_pool
        num_pages = 0 if sized is None else sized.size(0)
        num_pages_stream = 0 if self.k_pool_stream is None else self.k_pool_stream.size(0)
        self._c = _CPagedKV(_ptr(self.k_pool), _ptr(self.v_pool), _ptr(self.stats), _ptr(self.page_table),
                            _ptr(self.seq_lens), self.page_table.size(0), self.page_table.size(1), num_pages,
                            self.pool_heads, _ptr(self.k_pool_stream), _ptr(self.v_pool_stream),
                            _ptr(self.ring_table), num_pages_stream, self.kv_bits)
        return ctypes.byref(self._c)


# A decode step of a small batch is two or three calls of some ten microseconds of GPU work each, so the marshalling is kept to
# what a call cannot do without: addresses travel as plain integers (the argument types make pointers of them), the
# current stream is asked for as a handle, without the stream object around it, and the calls of the step itself are native.
def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("lserve binding takes contiguous tensors")
    return t.data_ptr()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # private names: the public way where they are gone
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream) -> int:
    if stream is None:
        if _raw_stream and _device and torch.cuda.is_initialized():
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, where: str) -> None:
    if rc:
        raise LserveError(rc, where)


def lserve_strerror(code: int) -> str:
    return load_library().lserve_strerror(int(code)).decode()


def lserve_last_hip_error() -> int:
    return int(load_library().lserve_last_hip_error())


def lserve_init() -> None:
    _check(load_library().lserve_init(), "lserve_init")


def lserve_workspace_bytes(which_call: int, desc: AttnDesc, batch: int = 0, max_pages_per_seq: int = 0,
                           sel_stride_or_budget_pages: int = 0, total_tokens: int = 0) -> int:
    return int(load_library().lserve_workspace_bytes(which_call, desc.c(), batch, max_pages_per_seq,
                                                     sel_stride_or_budget_pages, total_tokens))


def lserve_build_page_stats(desc: AttnDesc, kv: PagedKV, start_pos: Optional[torch.Tensor] = None,
                            max_tail_pages: int = 0, stream=None) -> None:
    _check(load_library().lserve_build_page_stats(desc.c(), kv.c(), _ptr(start_pos), max_tail_pages,
                                                  _stream(stream)), "lserve_build_page_stats")


def lserve_append_kv(desc: AttnDesc, kv: PagedKV, k_new: torch.Tensor, v_new: torch.Tensor, cu_new: torch.Tensor,
                     start_pos: torch.Tensor, max_new_per_seq: int, stream=None) -> None:
    _check((_calls or _native()).append(desc._address, kv, k_new, v_new, cu_new, start_pos, max_new_per_seq,
                                        _stream(stream)), "lserve_append_kv")


def lserve_select_pages(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, budget_tokens: int,
                        sel_pages: torch.Tensor, sel_count: torch.Tensor, sel_seq_len: torch.Tensor,
                        scores_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                        stream=None, stats_valid_len: Optional[torch.Tensor] = None) -> None:
    _check((_calls or _native()).select(desc._address, kv, q, budget_tokens, stats_valid_len, sel_pages, sel_count, sel_seq_len,
                                        scores_out, workspace, _stream(stream)), "lserve_select_pages")


def lserve_chunk_scratch_bytes(desc: AttnDesc, batch: int, total_new: int, max_new_per_seq: int, pages: int,
                               kv_bits: int = 16) -> int:
    return int(load_library().lserve_chunk_scratch_bytes(desc.c(), batch, total_new, max_new_per_seq, pages, kv_bits))


def _capture_has_a_pool() -> bool:
    """Under capture: do allocations come from a pool that the graph keeps (torch.cuda.graph), or from the one whose memory is handed
    on after the call and would be somebody else's when the graph is replayed (a capture begun by other means)?"""
    probe = torch.empty((16,), dtype=torch.uint8, device="cuda")
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= probe.data_ptr() < segment["address"] + segment["total_size"]:
            return tuple(segment.get("segment_pool_id", (0, 0))) != (0, 0)
    return False


def _chunk_scratch(desc: AttnDesc, q: torch.Tensor, batch: int, max_new_per_seq: int, pages: int, kv_bits: int,
                   stream) -> Optional[torch.Tensor]:
    """Scratch for a call on chunks, from torch's allocator, which hands freed memory on in the order of the stream it was taken on:
    it is taken on the stream of the call."""
    need = lserve_chunk_scratch_bytes(desc, batch, q.shape[0], max_new_per_seq, pages, kv_bits)
    if need == 0 or not q.is_cuda:
        return None
    handle = _stream(stream)
    on_stream = contextlib.nullcontext()
    if handle != _stream(None):
        if isinstance(stream, torch.cuda.Stream):
            on_stream = torch.cuda.stream(stream)
        elif handle == 0:
            on_stream = torch.cuda.stream(torch.cuda.default_stream(q.device))
        elif handle < 16:  # the runtime's names for streams are not addresses, as which torch would take them
            return None
        else:
            on_stream = torch.cuda.stream(torch.cuda.ExternalStream(handle, device=q.device))
    with on_stream:
        if torch.cuda.is_current_stream_capturing() and not _capture_has_a_pool():
            return None
        try:
            return torch.empty((need,), dtype=torch.uint8, device="cuda")
        except torch.cuda.OutOfMemoryError:
            warnings.warn(f"no memory for the {need} bytes of scratch of a call on chunks: it goes without, which is slower and adds "
                          "up in another order; scratch= takes memory of the caller's, an empty tensor for none",
                          RuntimeWarning, stacklevel=3)
            return None


def lserve_sparse_prefill(desc: AttnDesc, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                          cu_seqlens: torch.Tensor, max_seqlen: int, out: torch.Tensor,
                          lse_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                          stream=None) -> None:
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().lserve_sparse_prefill(desc.c(), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens),
                                                cu_seqlens.shape[0] - 1, q.shape[0], max_seqlen, _ptr(out),
                                                _ptr(lse_out), _ptr(workspace), ws_bytes, _stream(stream)),
           "lserve_sparse_prefill")


@dataclass
class BlockMask:
    """Mirror of lserve_block_mask (device int32 tensors); keeps the tensors alive."""
    head_mask: torch.Tensor
    q_tile_start: torch.Tensor
    row_ptr: torch.Tensor
    cols: Optional[torch.Tensor]
    num_masks: int
    rows_per_mask: int

    @property
    def nnz(self) -> int:
        return 0 if self.cols is None else int(self.cols.numel())

    def c(self):
        self._c = _CBlockMask(_ptr(self.head_mask), _ptr(self.q_tile_start), _ptr(self.row_ptr), _ptr(self.cols),
                              self.num_masks, self.rows_per_mask, self.nnz)
        return ctypes.byref(self._c)


def lserve_masked_prefill_workspace_bytes(desc: AttnDesc, batch: int, total_tokens: int, max_seqlen: int,
                                          num_masks: int, nnz: int) -> int:
    return int(load_library().lserve_masked_prefill_workspace_bytes(desc.c(), batch, total_tokens, max_seqlen,
                                                                    num_masks, nnz))


def lserve_sparse_prefill_masked(desc: AttnDesc, mask: BlockMask, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                                 cu_seqlens: torch.Tensor, max_seqlen: int, out: torch.Tensor,
                                 lse_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                 stream=None) -> None:
    ws_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(load_library().lserve_sparse_prefill_masked(desc.c(), mask.c(), _ptr(q), _ptr(k), _ptr(v),
                                                       _ptr(cu_seqlens), cu_seqlens.shape[0] - 1, q.shape[0],
                                                       max_seqlen, _ptr(out), _ptr(lse_out), _ptr(workspace),
                                                       ws_bytes, _stream(stream)),
           "lserve_sparse_prefill_masked")


def lserve_paged_prefill_workspace_bytes(desc: AttnDesc, batch: int, max_pages_per_seq: int) -> int:
    return int(load_library().lserve_paged_prefill_workspace_bytes(desc.c(), batch, max_pages_per_seq))


def lserve_sparse_prefill_paged(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, cu_q: torch.Tensor,
                                max_new_per_seq: int, max_seqlen: int, out: torch.Tensor,
                                lse_out: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None,
                                stream=None, scratch: Optional[torch.Tensor] = None) -> None:
    """workspace is not used.  scratch: see lserve_sparse_prefill_chunk; lserve_chunk_scratch_bytes with
    pages = min(page_table.shape[1], ceil(max_seqlen / 64))."""
    _ptr(workspace)  # unused, and contiguous all the same
    if scratch is None:
        pages = min(kv.page_table.shape[1], (max_seqlen - 1) // 64 + 1)
        scratch = _chunk_scratch(desc, q, cu_q.shape[0] - 1, max_new_per_seq, pages, 16, stream)
    _check(load_library().lserve_sparse_prefill_paged_scratch(
        desc.c(), kv.c(), _ptr(q), _ptr(cu_q), q.shape[0], max_new_per_seq, max_seqlen, _ptr(out), _ptr(lse_out), _ptr(scratch),
        0 if scratch is None else scratch.numel() * scratch.element_size(), _stream(stream)), "lserve_sparse_prefill_paged")


def lserve_sparse_prefill_chunk(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                                cu_new: torch.Tensor, max_new_per_seq: int, out: torch.Tensor,
                                lse_out: Optional[torch.Tensor] = None, stream=None,
                                scratch: Optional[torch.Tensor] = None) -> None:
    """scratch: device memory of lserve_chunk_scratch_bytes(desc, batch, q.shape[0], max_new_per_seq, page_table.shape[1], kv_bits)
    bytes or more, not shared with work in flight; too little of it, an empty tensor for instance: the call does without.  None: taken
    from torch's allocator for the call (up to 1 GiB of expanded pages, by the width of the page table, and 34 to 136 MB of pieces),
    on whatever stream it goes to and from the graph's own pool under torch.cuda.graph, so that the same call gives the same bits
    everywhere.  A call goes without, slower and with sums in another order, where torch is out of memory (a RuntimeWarning says
    so) and in a capture begun by other means than torch.cuda.graph."""
    if scratch is None:
        scratch = _chunk_scratch(desc, q, cu_new.shape[0] - 1, max_new_per_seq, kv.page_table.shape[1], kv.kv_bits, stream)
    _check(load_library().lserve_sparse_prefill_chunk_scratch(
        desc.c(), kv.c(), _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(cu_new), q.shape[0], max_new_per_seq, _ptr(out),
        _ptr(lse_out), _ptr(scratch), 0 if scratch is None else scratch.numel() * scratch.element_size(), _stream(stream)),
        "lserve_sparse_prefill_chunk")


def lserve_sparse_decode(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, sel_pages: Optional[torch.Tensor],
                         sel_count: Optional[torch.Tensor], sel_seq_len: Optional[torch.Tensor],
                         out: torch.Tensor, lse_out: Optional[torch.Tensor] = None,
                         workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    _check((_calls or _native()).decode(desc._address, kv, q, sel_pages, sel_count, sel_seq_len, out, lse_out, workspace,
                                        _stream(stream)), "lserve_sparse_decode")


def lserve_sparse_decode_noalloc(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, sel_pages: Optional[torch.Tensor],
                                 sel_count: Optional[torch.Tensor], sel_seq_len: Optional[torch.Tensor],
                                 out: torch.Tensor, lse_out: Optional[torch.Tensor] = None, stream=None) -> None:
    sel_stride = 0 if sel_pages is None else sel_pages.shape[-1]
    _check(load_library().lserve_sparse_decode_noalloc(desc.c(), kv.c(), _ptr(q), _ptr(sel_pages), _ptr(sel_count),
                                                       _ptr(sel_seq_len), sel_stride, _ptr(out), _ptr(lse_out),
                                                       _stream(stream)), "lserve_sparse_decode_noalloc")


def lserve_probe_decode_read(desc: AttnDesc, kv: PagedKV, sel_pages: Optional[torch.Tensor],
                             sel_count: Optional[torch.Tensor], sel_seq_len: Optional[torch.Tensor], stream=None) -> None:
    sel_stride = 0 if sel_pages is None else sel_pages.shape[-1]
    _check(load_library().lserve_probe_decode_read(desc.c(), kv.c(), _ptr(sel_pages), _ptr(sel_count), _ptr(sel_seq_len),
                                                   sel_stride, _stream(stream)), "lserve_probe_decode_read")


def lserve_probe_prefill_shape(desc: AttnDesc, batch: int, total_rows: int, max_rows: int, pages: int = 0,
                               kv_bits: int = 16) -> tuple:
    """(key slices, dense heads folded, streaming heads folded, units are query tiles of one head) of a prefill launch."""
    shape = (ctypes.c_int32 * 4)()
    _check(load_library().lserve_probe_prefill_shape(desc.c(), batch, total_rows, max_rows, pages, kv_bits, shape),
           "lserve_probe_prefill_shape")
    return tuple(shape)


def lserve_probe_prefill_plan(desc: AttnDesc, batch: int, total_rows: int, max_rows: int, pages: int = 0, kv_bits: int = 16,
                              scratch: bool = True) -> dict:
    """The rest of it: key ranges of a dense and of a streaming head's rows, half workgroups, pieces, streaming heads in the launch
    that puts pieces together, expanded pages."""
    plan = (ctypes.c_int32 * 6)()
    _check(load_library().lserve_probe_prefill_plan(desc.c(), batch, total_rows, max_rows, pages, kv_bits, int(scratch), plan),
           "lserve_probe_prefill_plan")
    return dict(zip(("dense", "streaming", "half", "pieces", "apart", "expand"), plan))


def lserve_probe_prefill_longest_first(desc: AttnDesc, batch: int, total_rows: int, max_rows: int) -> bool:
    """Prompts: has the first workgroup of every compute unit, with the longest walks, the higher wave priority?"""
    first = ctypes.c_int32()
    _check(load_library().lserve_probe_prefill_longest_first(desc.c(), batch, total_rows, max_rows, ctypes.byref(first)),
           "lserve_probe_prefill_longest_first")
    return bool(first.value)


def lserve_probe_mask_walk(desc: AttnDesc, batch: int, total_tokens: int, max_seqlen: int, num_masks: int, rows_per_mask: int,
                           nnz: int) -> int:
    """How a masked prefill walks its lists: 0 merged, 1 by rows in four key slices, 2 by rows in half workgroups."""
    walk = ctypes.c_int32()
    _check(load_library().lserve_probe_mask_walk(desc.c(), batch, total_tokens, max_seqlen, num_masks, rows_per_mask, nnz,
                                                 ctypes.byref(walk)), "lserve_probe_mask_walk")
    return walk.value


def lserve_extend_tables(desc: AttnDesc, kv: PagedKV, new_lens: torch.Tensor, free_pages: Optional[torch.Tensor], cu_new: torch.Tensor,
                         new_seq_lens: torch.Tensor, pages_taken: torch.Tensor, positions: Optional[torch.Tensor] = None,
                         slots: Optional[torch.Tensor] = None, ring_slots: Optional[torch.Tensor] = None, stream=None,
                         total_new: Optional[int] = None) -> None:
    """total_new: new tokens of the batch or more, the length of positions, slots and ring_slots (and taken from the first of
    them that is given)."""
    if total_new is None:
        given = positions if positions is not None else slots if slots is not None else ring_slots
        if given is None:
            raise ValueError("lserve_extend_tables: total_new, where no positions or slots are asked for")
        total_new = given.numel()
    if total_new >= 2 ** 31:
        raise ValueError(f"lserve_extend_tables: {total_new} new tokens, more than 32 bits count")
    _check((_calls or _native()).extend(desc._address, kv, new_lens, free_pages, cu_new, new_seq_lens, pages_taken, positions, slots,
                                        ring_slots, total_new, _stream(stream)), "lserve_extend_tables")


_SCALINGS = ("none", "linear", "wavelength", "ramp")


def lserve_rotary_frequencies(rotary_dim: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                              original_positions: float = 8192.0, low: float = 1.0, high: float = 4.0) -> tuple:
    """(rotary_dim / 2 frequencies, radians per position, float64 on the host; factor on what turns)."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling is one of {_SCALINGS}")
    out = torch.empty((max(1, rotary_dim // 2),), dtype=torch.float64)
    loud = ctypes.c_float()
    c = _CRotaryScaling(_SCALINGS.index(scaling), rotary_dim, base, factor, original_positions, low, high)
    _check(load_library().lserve_rotary_frequencies(ctypes.byref(c), out.data_ptr(), ctypes.addressof(loud)), "lserve_rotary_frequencies")
    return out, loud.value


@dataclass
class RotaryDesc:
    """Mirror of lserve_rotary_desc: how the heads of a layer turn.  The frequencies are those of lserve_rotary_frequencies, or the
    caller's own (inv_freq: float64 [rotary_dim / 2], radians per position), kept on `device` (the current GPU); calls read inv_freq where it is
    by then."""
    rotary_dim: int = 128
    interleaved: bool = False
    base: float = 10000.0
    scaling: str = "none"
    factor: float = 1.0
    original_positions: float = 8192.0
    low: float = 1.0
    high: float = 4.0
    scale: float = 0.0  # 0: what the scaling gives
    inv_freq: Optional[torch.Tensor] = None
    device: Optional[object] = None

    def __post_init__(self):
        if self.inv_freq is None:
            self.inv_freq, loud = lserve_rotary_frequencies(self.rotary_dim, self.base, self.scaling, self.factor,
                                                            self.original_positions, self.low, self.high)
            self.scale = self.scale or loud
        if self.inv_freq.dtype != torch.float64 or self.inv_freq.numel() < self.rotary_dim // 2:
            raise ValueError("RotaryDesc: inv_freq holds rotary_dim / 2 numbers of 64 bits")
        where = self.device if self.device is not None else ("cuda" if torch.cuda.is_available() else "cpu")
        self.inv_freq = self.inv_freq.to(where).contiguous()
        self._c = _CRotaryDesc(self.rotary_dim, int(self.interleaved), self.inv_freq.data_ptr(), float(self.scale))

    def c(self):
        return ctypes.byref(self._c)

    @property
    def _address(self):
        return ctypes.addressof(self._c)


def lserve_rotary(desc: AttnDesc, rotary: RotaryDesc, q: Optional[torch.Tensor], k: Optional[torch.Tensor], positions: torch.Tensor,
                  q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor], stream=None) -> None:
    """q and k may be cut out of the rows of a fused projection (any distance between rows that is a multiple of eight elements)."""
    _check((_calls or _native()).rotary(desc._address, rotary._address, rotary.inv_freq, q, k, positions, q_out, k_out, _stream(stream)),
           "lserve_rotary")


@functools.lru_cache(maxsize=256)
def _axes_of_pairs(pairs: bytes):
    """The library's list of axes: it reads rotary_dim / 2 of them, 64 at most, and what is not named here is no axis.  Kept for the lists that a program has, so
    that a description made for a single call does not take its list with it."""
    axes = (ctypes.c_uint8 * max(64, len(pairs)))(*([255] * 64))
    axes[:len(pairs)] = pairs
    return axes


class PositionAxes:
    """Mirror of lserve_position_axes: the axis of each of a head's rotary_dim / 2 pairs (num_axes: as many as are named).  Stays as it was made."""

    def __init__(self, pair_axis: Sequence[int], num_axes: int = 0):
        pairs = [int(a) for a in pair_axis]
        if not pairs or min(pairs) < 0 or max(pairs) > 255:
            raise ValueError("PositionAxes: an axis for every pair")
        self._pairs, self._axes = len(pairs), _axes_of_pairs(bytes(pairs))
        self._c = _CPositionAxes(num_axes or max(pairs) + 1, ctypes.cast(self._axes, ctypes.POINTER(ctypes.c_uint8)))
        self._address = ctypes.addressof(self._c)

    @property
    def pair_axis(self) -> list:
        return list(self._axes[:self._pairs])

    @property
    def num_axes(self) -> int:
        return self._c.num_axes

    def __eq__(self, other):
        return isinstance(other, PositionAxes) and (self.pair_axis, self.num_axes) == (other.pair_axis, other.num_axes)

    __hash__ = None

    def __repr__(self):
        return f"PositionAxes(pair_axis={self.pair_axis}, num_axes={self.num_axes})"

    @classmethod
    def sections(cls, *pairs: int) -> "PositionAxes":
        """The first pairs[0] pairs turn by axis 0, the next pairs[1] by axis 1, ..."""
        return cls([a for a, n in enumerate(pairs) for _ in range(n)], len(pairs))

    @classmethod
    def in_turn(cls, *pairs: int) -> "PositionAxes":
        """Axis a > 0 has pairs a, a + A, a + 2 A, ..., pairs[a] of A axes' in all, axis 0 the others (of sum(pairs))."""
        n, axes = sum(pairs), len(pairs)
        if any(m and a + (m - 1) * axes >= n for a, m in enumerate(pairs) if a):
            raise ValueError(f"PositionAxes: {pairs} pairs do not go in turn")
        return cls([i % axes if i // axes < pairs[i % axes] else 0 for i in range(n)], axes)


@dataclass
class HeadNorm:
    """Mirror of lserve_head_norm; weights: float32 [D] for all heads, or [heads][D] (both alike), or None for ones.  A call works with what
    the attributes are by then, and with the memory that the weights' tensors have by then."""
    q_weight: Optional[torch.Tensor] = None
    k_weight: Optional[torch.Tensor] = None
    eps: float = 1e-6
    centred: bool = False

    def __setattr__(self, name, value):
        described = "_c" in self.__dict__ and name in self.__dataclass_fields__
        before = getattr(self, name, None)
        super().__setattr__(name, value)
        if described:
            try:
                self.__post_init__()
            except ValueError:
                super().__setattr__(name, before)
                raise

    def __post_init__(self):
        given = [w for w in (self.q_weight, self.k_weight) if w is not None]
        if any(w.dtype != torch.float32 or w.dim() not in (1, 2) or w.dim() != given[0].dim() for w in given):
            raise ValueError("HeadNorm: weights are [D] or [heads][D], of 32 bits")
        self._c = _CHeadNorm(int(self.centred), int(bool(given) and given[0].dim() == 2), float(self.eps), _ptr(self.q_weight), _ptr(self.k_weight))
        self._address = ctypes.addressof(self._c)


def lserve_rotary_axes(desc: AttnDesc, rotary: RotaryDesc, axes: PositionAxes, q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                       positions: torch.Tensor, q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor], stream=None) -> None:
    """positions: int32 [axes][total], axes any distance apart; q and k as in lserve_rotary."""
    if positions is None:
        raise ValueError("lserve_rotary_axes: positions [axes][total]")
    _check((_calls or _native()).turned(desc._address, 0, rotary._address, axes._address, None, None, rotary.inv_freq, q, k, positions, q_out,
                                        k_out, _stream(stream)), "lserve_rotary_axes")


def lserve_norm_rotary(desc: AttnDesc, norm: HeadNorm, rotary: Optional[RotaryDesc], q: Optional[torch.Tensor], k: Optional[torch.Tensor],
                       positions: Optional[torch.Tensor], q_out: Optional[torch.Tensor], k_out: Optional[torch.Tensor], stream=None,
                       axes: Optional[PositionAxes] = None) -> None:
    """positions: int32 [total], with axes [axes][total]; without rotary None will do."""
    _check((_calls or _native()).turned(desc._address, norm._address, rotary._address if rotary else 0, axes._address if axes else 0, norm.q_weight,
                                        norm.k_weight, rotary.inv_freq if rotary else None, q, k, positions, q_out, k_out, _stream(stream)),
           "lserve_norm_rotary")


def lserve_rotary_append_kv(desc: AttnDesc, kv: PagedKV, rotary: Optional[RotaryDesc], q: Optional[torch.Tensor], k: torch.Tensor,
                            v: torch.Tensor, cu_new: torch.Tensor, start_pos: torch.Tensor, max_new_per_seq: int, q_out: Optional[torch.Tensor],
                            k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None, norm: Optional[HeadNorm] = None,
                            axes: Optional[PositionAxes] = None, positions: Optional[torch.Tensor] = None, stream=None) -> None:
    """positions: int32 [total_new], with axes [axes][total_new], or None: start_pos[b] + j.  q, k and v may be cut out of the rows of a fused
    projection."""
    _check((_calls or _native()).rotary_append(
        desc._address, kv, norm._address if norm else 0, rotary._address if rotary else 0, axes._address if axes else 0, norm.q_weight if norm else None,
        norm.k_weight if norm else None, rotary.inv_freq if rotary else None, q, k, v, positions, cu_new, start_pos, max_new_per_seq, q_out, k_out, v_out,
        _stream(stream)), "lserve_rotary_append_kv")


def lserve_tree_masks(parents: torch.Tensor, cu_new: torch.Tensor, seq_lens: torch.Tensor, max_new_per_seq: int,
                      tree_mask: torch.Tensor, positions: torch.Tensor, stream=None) -> None:
    """tree_mask: int64 [total_new][words], 64 drafted tokens to a word."""
    _check((_calls or _native()).masks(parents, cu_new, seq_lens, max_new_per_seq, tree_mask, positions, _stream(stream)), "lserve_tree_masks")


def lserve_tree_workspace_bytes(desc: AttnDesc, batch: int, total_new: int, max_new_per_seq: int, max_pages_per_seq: int,
                                sel_stride: int = 0) -> int:
    """For a call of just these sizes; smaller ones may need more (a workspace kept for many: the largest over them, or
    LSERVE_TREE_WORKSPACE_MOST)."""
    return int(load_library().lserve_tree_workspace_bytes(desc.c(), batch, total_new, max_new_per_seq, max_pages_per_seq, sel_stride))


def lserve_sparse_decode_tree(desc: AttnDesc, kv: PagedKV, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                              cu_new: torch.Tensor, max_new_per_seq: int, out: torch.Tensor, lse_out: Optional[torch.Tensor] = None,
                              tree_mask: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                              sel_pages: Optional[torch.Tensor] = None, sel_count: Optional[torch.Tensor] = None,
                              sel_seq_len: Optional[torch.Tensor] = None, workspace: Optional[torch.Tensor] = None, stream=None) -> None:
    """tree_mask: int64 [total_new][words], 64 drafted tokens to a word; without it and positions the drafted tokens are a chain.
    Without sel_pages, sel_count and sel_seq_len selecting heads attend the whole history."""
    _check((_calls or _native()).tree(desc._address, kv, q, k_new, v_new, cu_new, max_new_per_seq, out, lse_out, tree_mask, positions,
                                      sel_pages, sel_count, sel_seq_len, workspace, _stream(stream)), "lserve_sparse_decode_tree")
