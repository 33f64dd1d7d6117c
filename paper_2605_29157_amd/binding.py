"""Thin ctypes binding of the Parallax HIP library (same names as include/parallax.h).

Only argument marshalling happens here: torch tensors supply device pointers, strides and the
current HIP stream; every step of the attention path runs in the library's kernels. There is
no CPU or PyTorch fallback: if the library is missing, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch  # imported before the library so both share one HIP runtime

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libparallax_hip.so")

PLX_BF16, PLX_F32 = 0, 1
PLX_MAX_SPLITS = 128
(PLX_OK, PLX_ERR_NULL, PLX_ERR_SHAPE, PLX_ERR_DTYPE, PLX_ERR_ALIGN, PLX_ERR_WORKSPACE,
 PLX_ERR_LAUNCH, PLX_ERR_SPLITS, PLX_ERR_SCALE, PLX_ERR_SCRATCH) = (0, -1, -2, -3, -4, -5, -6, -7, -8, -9)
PLX_STATIC_SCRATCH_RECORDS = 16384

EXPORTED_SYMBOLS = (
    "parallax_decode_workspace_bytes", "parallax_decode_num_splits", "parallax_decode_call_splits", "parallax_decode",
    "parallax_decode_partials", "parallax_decode_combine", "parallax_decode_fused",
    "parallax_decode_static", "parallax_decode_static_scratch_bytes",
    "parallax_decode_sinks", "parallax_decode_sinks_call_splits", "parallax_decode_tree", "parallax_decode_tree_call_splits",
    "parallax_decode_mla", "parallax_decode_mla_workspace_bytes", "parallax_decode_mla_num_splits",
    "parallax_prefill", "parallax_prefill_split", "parallax_prefill_workspace_bytes", "parallax_prefill_form", "parallax_prefill_backward", "parallax_prefill_backward_form",
    "parallax_prefill_backward_workspace_bytes",
    "parallax_prefill_sinks", "parallax_prefill_backward_sinks", "parallax_prefill_backward_sinks_workspace_bytes",
    "parallax_q4_row_bytes", "parallax_cache_write_q4", "parallax_cache_read_q4", "parallax_decode_q4",
    "parallax_decode_q4_call_splits", "parallax_cache_bounds", "parallax_select_blocks",
    "parallax_select_blocks_workspace_bytes", "parallax_decode_blocks", "parallax_decode_blocks_call_splits",
    "parallax_cache_fork", "parallax_cache_extend", "parallax_cache_free", "parallax_cache_copy", "parallax_cache_compact",
    "parallax_block_lists", "parallax_norm_rope", "parallax_rope_table", "parallax_util_copy", "parallax_util_read",
    "parallax_util_read_grid", "parallax_util_read_sink_slots", "parallax_util_mfma", "parallax_strerror", "parallax_version",
)


class plx_qr_prep(ctypes.Structure):
    _fields_ = [("q_gamma", ctypes.c_void_p), ("r_gamma", ctypes.c_void_p), ("rope_table", ctypes.c_void_p),
                ("pos0", ctypes.c_void_p), ("rope_positions", ctypes.c_int32), ("rope_q", ctypes.c_int32),
                ("rope_r", ctypes.c_int32), ("eps", ctypes.c_float)]


class plx_decode_args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("r", ctypes.c_void_p),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("o", ctypes.c_void_p),
        ("seq_lens", ctypes.c_void_p),
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
        ("Lmax", ctypes.c_int32), ("d", ctypes.c_int32),
        ("k_stride_b", ctypes.c_int64), ("k_stride_h", ctypes.c_int64), ("k_stride_l", ctypes.c_int64),
        ("v_stride_b", ctypes.c_int64), ("v_stride_h", ctypes.c_int64), ("v_stride_l", ctypes.c_int64),
        ("scale", ctypes.c_float),
        ("use_r", ctypes.c_int32),
        ("num_splits", ctypes.c_int32),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("dtype", ctypes.c_int),
        ("block_table", ctypes.c_void_p),
        ("page_size", ctypes.c_int32), ("block_table_stride", ctypes.c_int32),
        ("num_pages", ctypes.c_int32),
        ("Tq", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("split_counters", ctypes.c_void_p),
        ("prep", plx_qr_prep),
    ]


class plx_decode_tree_args(ctypes.Structure):
    _fields_ = [("decode", plx_decode_args), ("tree_mask", ctypes.c_void_p), ("draft_lens", ctypes.c_void_p),
                ("mask_batch", ctypes.c_int32), ("sinks", ctypes.c_int32)]


class plx_prefill_args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("r", ctypes.c_void_p),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("o", ctypes.c_void_p),
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
        ("T", ctypes.c_int32), ("d", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("r_stride", ctypes.c_int64 * 3),
        ("k_stride", ctypes.c_int64 * 3), ("v_stride", ctypes.c_int64 * 3),
        ("o_stride", ctypes.c_int64 * 3),
        ("scale", ctypes.c_float),
        ("causal", ctypes.c_int32),
        ("use_r", ctypes.c_int32),
        ("dtype", ctypes.c_int),
        ("Tkv", ctypes.c_int32),
        ("window", ctypes.c_int32),
        ("vbar", ctypes.c_void_p), ("row_stats", ctypes.c_void_p),
        ("sparse_row_ptr", ctypes.c_void_p), ("sparse_tile_idx", ctypes.c_void_p),
        ("sparse_batch", ctypes.c_int32), ("sparse_heads", ctypes.c_int32),
        ("prep", plx_qr_prep),
    ]


class plx_prefill_bwd_args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("r", ctypes.c_void_p),
        ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
        ("o", ctypes.c_void_p), ("vbar", ctypes.c_void_p),
        ("row_stats", ctypes.c_void_p),
        ("d_o", ctypes.c_void_p),
        ("dq", ctypes.c_void_p), ("dr", ctypes.c_void_p),
        ("dk", ctypes.c_void_p), ("dv", ctypes.c_void_p),
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
        ("T", ctypes.c_int32), ("Tkv", ctypes.c_int32), ("d", ctypes.c_int32),
        ("scale", ctypes.c_float),
        ("causal", ctypes.c_int32),
        ("dtype", ctypes.c_int), ("window", ctypes.c_int32),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("q_stride", ctypes.c_int64 * 3), ("r_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3), ("o_stride", ctypes.c_int64 * 3), ("vbar_stride", ctypes.c_int64 * 3),
        ("d_o_stride", ctypes.c_int64 * 3), ("dq_stride", ctypes.c_int64 * 3), ("dr_stride", ctypes.c_int64 * 3),
        ("dk_stride", ctypes.c_int64 * 3), ("dv_stride", ctypes.c_int64 * 3),
        ("sparse_row_ptr", ctypes.c_void_p), ("sparse_tile_idx", ctypes.c_void_p),
        ("sparse_col_ptr", ctypes.c_void_p), ("sparse_col_idx", ctypes.c_void_p),
        ("sparse_batch", ctypes.c_int32), ("sparse_heads", ctypes.c_int32),
    ]


class plx_decode_mla_args(ctypes.Structure):
    _fields_ = [
        ("q", ctypes.c_void_p), ("r", ctypes.c_void_p), ("ckv", ctypes.c_void_p), ("o", ctypes.c_void_p),
        ("seq_lens", ctypes.c_void_p),
        ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Lmax", ctypes.c_int32),
        ("d_latent", ctypes.c_int32), ("d_rope", ctypes.c_int32), ("num_splits", ctypes.c_int32),
        ("ckv_stride_b", ctypes.c_int64), ("ckv_stride_l", ctypes.c_int64),
        ("scale", ctypes.c_float), ("dtype", ctypes.c_int),
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
        ("block_table", ctypes.c_void_p),
        ("page_size", ctypes.c_int32), ("num_pages", ctypes.c_int32), ("block_table_stride", ctypes.c_int32),
        ("Tq", ctypes.c_int32), ("window", ctypes.c_int32),
    ]


class plx_block_list_args(ctypes.Structure):
    _fields_ = [("mask", ctypes.c_void_p), ("lists", ctypes.c_int32), ("n_row_blocks", ctypes.c_int32),
                ("n_tiles", ctypes.c_int32), ("counts", ctypes.c_void_p), ("row_ptr", ctypes.c_void_p),
                ("tile_idx", ctypes.c_void_p), ("col_ptr", ctypes.c_void_p), ("col_idx", ctypes.c_void_p)]


class plx_page_table(ctypes.Structure):
    _fields_ = [("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p), ("page_refs", ctypes.c_void_p),
                ("free_pages", ctypes.c_void_p), ("free_count", ctypes.c_void_p), ("sequences", ctypes.c_int32),
                ("pages_per_sequence", ctypes.c_int32), ("block_table_stride", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("page_size", ctypes.c_int32)]


class plx_cache_pools(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("num_pages", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("d", ctypes.c_int32), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("dtype", ctypes.c_int)]


class plx_cache_compact_args(ctypes.Structure):
    _fields_ = [("pools", plx_cache_pools), ("block_table", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
                ("draft_lens", ctypes.c_void_p), ("accepted", ctypes.c_void_p), ("n_accepted", ctypes.c_void_p),
                ("new_lens", ctypes.c_void_p), ("B", ctypes.c_int32), ("block_table_stride", ctypes.c_int32),
                ("max_draft", ctypes.c_int32), ("max_accepted", ctypes.c_int32)]


class plx_q4_cache(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_void_p), ("stride", ctypes.c_int64 * 3), ("block_table", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("block_table_stride", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("B", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("capacity", ctypes.c_int32), ("d", ctypes.c_int32)]


class plx_q4_rows_args(ctypes.Structure):
    _fields_ = [("cache", plx_q4_cache), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("start", ctypes.c_void_p), ("counts", ctypes.c_void_p),
                ("T", ctypes.c_int32), ("dtype", ctypes.c_int)]


class plx_cache_bounds_args(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3), ("block_table", ctypes.c_void_p),
                ("page_size", ctypes.c_int32), ("block_table_stride", ctypes.c_int32), ("num_pages", ctypes.c_int32),
                ("B", ctypes.c_int32), ("Hkv", ctypes.c_int32), ("capacity", ctypes.c_int32), ("d", ctypes.c_int32),
                ("q4", ctypes.c_void_p), ("bounds", ctypes.c_void_p), ("n_blocks", ctypes.c_int32),
                ("max_new", ctypes.c_int32), ("seq_lens", ctypes.c_void_p), ("from_lens", ctypes.c_void_p)]


class plx_select_blocks_args(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("bounds", ctypes.c_void_p), ("seq_lens", ctypes.c_void_p),
                ("block_list", ctypes.c_void_p), ("B", ctypes.c_int32), ("Hq", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("Tq", ctypes.c_int32), ("d", ctypes.c_int32), ("n_blocks", ctypes.c_int32), ("keep", ctypes.c_int32),
                ("first", ctypes.c_int32), ("recent", ctypes.c_int32), ("workspace", ctypes.c_void_p),
                ("workspace_bytes", ctypes.c_size_t)]


class plx_decode_blocks_args(ctypes.Structure):
    _fields_ = [("decode", plx_decode_args), ("block_list", ctypes.c_void_p), ("n_list", ctypes.c_int32)]


class plx_decode_q4_args(ctypes.Structure):
    _fields_ = [("decode", plx_decode_args), ("cache", plx_q4_cache), ("sinks", ctypes.c_int32), ("n_list", ctypes.c_int32),
                ("block_list", ctypes.c_void_p)]


class plx_norm_rope_tensor(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("gamma", ctypes.c_void_p),
                ("H", ctypes.c_int32), ("rope", ctypes.c_int32)]


class plx_norm_rope_args(ctypes.Structure):
    _fields_ = [("tensors", plx_norm_rope_tensor * 3), ("n_tensors", ctypes.c_int32),
                ("B", ctypes.c_int32), ("T", ctypes.c_int32), ("d", ctypes.c_int32),
                ("pos0", ctypes.c_void_p), ("eps", ctypes.c_float), ("theta", ctypes.c_float),
                ("dtype", ctypes.c_int), ("rope_table", ctypes.c_void_p), ("table_positions", ctypes.c_int32)]


# The same layouts for struct.pack: a call fills its arguments in one go (30 - 60 assignments of
# ctypes fields and arrays cost 4 - 12 us of host time, as much as a small step takes on the GPU).
_PREP = "4P3if"
_PACK = {
    plx_decode_args: struct.Struct("@6P5i6qf2iPNiP3i2iP" + _PREP + "0P"),
    plx_prefill_args: struct.Struct("@5P5i15qf5i2P2P2i" + _PREP + "0P"),
    plx_prefill_bwd_args: struct.Struct("@12P6if3iPN33q4P2i0P"),
    plx_decode_mla_args: struct.Struct("@5P3i3i2qfiPNP3i2i0P"),
    plx_norm_rope_args: struct.Struct("@" + 3 * "3P2i" + "4iP2fiPi0P"),
    plx_block_list_args: struct.Struct("@P3i5P"),
    plx_page_table: struct.Struct("@5P5i0P"),
    plx_cache_pools: struct.Struct("@2P4i6qi0P"),
    plx_cache_compact_args: struct.Struct("@2P4i6qi0P6P4i0P"),
    plx_q4_cache: struct.Struct("@P3qP7i0P"),
    plx_q4_rows_args: struct.Struct("@P3qP7i0P2P6q2P2i0P"),
    plx_cache_bounds_args: struct.Struct("@P3qP7i2P2i2P"),
    plx_select_blocks_args: struct.Struct("@4P9iPN0P"),
    plx_decode_blocks_args: struct.Struct("@6P5i6qf2iPNiP3i2iP" + _PREP + "0PPi0P"),
    plx_decode_q4_args: struct.Struct("@6P5i6qf2iPNiP3i2iP" + _PREP + "0PP3qP7i0P2iP"),
}
for _args, _format in _PACK.items():
    assert _format.size == ctypes.sizeof(_args), _args
_NO_PREP = (0,) * 8
_ROW_LISTS, _ALL_LISTS = struct.Struct("@2P2i"), struct.Struct("@4P2i")  # from sparse_row_ptr on
_ROW_CACHE = struct.Struct("@2P")  # from vbar on


def _filled(args, *values):
    return args.from_buffer_copy(_PACK[args].pack(*values))


def _f32(x) -> float:  # (as a C float takes it: too large becomes infinite, not an error here)
    return x if type(x) is float and -3.4e38 < x < 3.4e38 else ctypes.c_float(float(x)).value


def _i32(x) -> int:  # (as a C int takes it)
    return x if type(x) is int and -0x80000000 <= x < 0x80000000 else ctypes.c_int32(int(x)).value


class ParallaxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__("%s failed: %s (status %d)" % (where, strerror(status), status))


_lib = None


def load_library() -> ctypes.CDLL:
    """Load libparallax_hip.so (built by __graft_entry__.build()). Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "%s is missing: build it with `python -c 'import __graft_entry__ as g; "
                "g.build()'` (there is no fallback path)" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        lib.parallax_decode_workspace_bytes.argtypes = [ctypes.c_int32] * 5
        lib.parallax_decode_workspace_bytes.restype = ctypes.c_size_t
        lib.parallax_decode_num_splits.argtypes = [ctypes.c_int32] * 6
        lib.parallax_decode_num_splits.restype = ctypes.c_int32
        lib.parallax_decode_call_splits.argtypes = [ctypes.POINTER(plx_decode_args)]
        lib.parallax_decode_call_splits.restype = ctypes.c_int32
        lib.parallax_decode.argtypes = [ctypes.POINTER(plx_decode_args), ctypes.c_void_p]
        lib.parallax_decode.restype = ctypes.c_int
        lib.parallax_decode_static_scratch_bytes.argtypes = []
        lib.parallax_decode_static_scratch_bytes.restype = ctypes.c_size_t
        for name in ("parallax_decode_partials", "parallax_decode_combine", "parallax_decode_fused",
                     "parallax_decode_static"):
            getattr(lib, name).argtypes = [ctypes.POINTER(plx_decode_args), ctypes.c_void_p]
            getattr(lib, name).restype = ctypes.c_int
        lib.parallax_decode_sinks.argtypes = [ctypes.POINTER(plx_decode_args), ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_decode_sinks.restype = ctypes.c_int
        lib.parallax_decode_sinks_call_splits.argtypes = [ctypes.POINTER(plx_decode_args), ctypes.c_int32]
        lib.parallax_decode_sinks_call_splits.restype = ctypes.c_int32
        lib.parallax_decode_tree.argtypes = [ctypes.POINTER(plx_decode_tree_args), ctypes.c_void_p]
        lib.parallax_decode_tree.restype = ctypes.c_int
        lib.parallax_decode_tree_call_splits.argtypes = [ctypes.POINTER(plx_decode_tree_args)]
        lib.parallax_decode_tree_call_splits.restype = ctypes.c_int32
        lib.parallax_prefill.argtypes = [ctypes.POINTER(plx_prefill_args), ctypes.c_void_p]
        lib.parallax_prefill.restype = ctypes.c_int
        lib.parallax_prefill_workspace_bytes.argtypes = [ctypes.POINTER(plx_prefill_args)]
        lib.parallax_prefill_workspace_bytes.restype = ctypes.c_size_t
        lib.parallax_prefill_form.argtypes = [ctypes.POINTER(plx_prefill_args), ctypes.c_size_t]
        lib.parallax_prefill_form.restype = ctypes.c_int32
        lib.parallax_prefill_split.argtypes = [ctypes.POINTER(plx_prefill_args), ctypes.c_void_p, ctypes.c_size_t,
                                               ctypes.c_void_p]
        lib.parallax_prefill_split.restype = ctypes.c_int
        lib.parallax_prefill_backward.argtypes = [ctypes.POINTER(plx_prefill_bwd_args), ctypes.c_void_p]
        lib.parallax_prefill_backward.restype = ctypes.c_int
        lib.parallax_prefill_backward_form.argtypes = [ctypes.POINTER(plx_prefill_bwd_args)]
        lib.parallax_prefill_backward_form.restype = ctypes.c_int32
        lib.parallax_prefill_backward_workspace_bytes.argtypes = [ctypes.c_int32] * 3
        lib.parallax_prefill_backward_workspace_bytes.restype = ctypes.c_size_t
        lib.parallax_block_lists.argtypes = [ctypes.POINTER(plx_block_list_args), ctypes.c_void_p]
        lib.parallax_block_lists.restype = ctypes.c_int
        lib.parallax_prefill_sinks.argtypes = [ctypes.POINTER(plx_prefill_args), ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_prefill_sinks.restype = ctypes.c_int
        lib.parallax_prefill_backward_sinks.argtypes = [ctypes.POINTER(plx_prefill_bwd_args), ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_prefill_backward_sinks.restype = ctypes.c_int
        lib.parallax_prefill_backward_sinks_workspace_bytes.argtypes = [ctypes.POINTER(plx_prefill_bwd_args), ctypes.c_int32]
        lib.parallax_prefill_backward_sinks_workspace_bytes.restype = ctypes.c_size_t
        _list = ctypes.c_void_p
        lib.parallax_cache_fork.argtypes = [ctypes.POINTER(plx_page_table), _list, _list, ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_cache_extend.argtypes = [ctypes.POINTER(plx_page_table), _list, _list, ctypes.c_int32, _list, _list, _list,
                                              _list, ctypes.c_void_p]
        lib.parallax_cache_free.argtypes = [ctypes.POINTER(plx_page_table), _list, _list, _list, ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_cache_copy.argtypes = [ctypes.POINTER(plx_cache_pools), _list, _list, _list, ctypes.c_int32, ctypes.c_void_p]
        lib.parallax_cache_compact.argtypes = [ctypes.POINTER(plx_cache_compact_args), ctypes.c_void_p]
        for name in ("fork", "extend", "free", "copy", "compact"):
            getattr(lib, "parallax_cache_" + name).restype = ctypes.c_int
        lib.parallax_q4_row_bytes.argtypes = [ctypes.c_int32]
        lib.parallax_q4_row_bytes.restype = ctypes.c_int32
        lib.parallax_select_blocks_workspace_bytes.argtypes = [ctypes.c_int32] * 3
        lib.parallax_select_blocks_workspace_bytes.restype = ctypes.c_size_t
        for name, args in (("parallax_cache_write_q4", plx_q4_rows_args), ("parallax_cache_read_q4", plx_q4_rows_args),
                           ("parallax_cache_bounds", plx_cache_bounds_args), ("parallax_select_blocks", plx_select_blocks_args),
                           ("parallax_decode_blocks", plx_decode_blocks_args), ("parallax_decode_q4", plx_decode_q4_args)):
            getattr(lib, name).argtypes = [ctypes.POINTER(args), ctypes.c_void_p]
            getattr(lib, name).restype = ctypes.c_int
        for name, args in (("parallax_decode_blocks", plx_decode_blocks_args), ("parallax_decode_q4", plx_decode_q4_args)):
            getattr(lib, name + "_call_splits").argtypes = [ctypes.POINTER(args)]
            getattr(lib, name + "_call_splits").restype = ctypes.c_int32
        lib.parallax_norm_rope.argtypes = [ctypes.POINTER(plx_norm_rope_args), ctypes.c_void_p]
        lib.parallax_norm_rope.restype = ctypes.c_int
        lib.parallax_rope_table.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32, ctypes.c_float,
                                            ctypes.c_void_p]
        lib.parallax_rope_table.restype = ctypes.c_int
        lib.parallax_util_copy.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t,
                                           ctypes.c_void_p]
        lib.parallax_util_copy.restype = ctypes.c_int
        lib.parallax_util_read.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p,
                                           ctypes.c_void_p]
        lib.parallax_util_read.restype = ctypes.c_int
        lib.parallax_util_read_grid.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p, ctypes.c_int32,
                                                ctypes.c_void_p]
        lib.parallax_util_read_grid.restype = ctypes.c_int
        lib.parallax_decode_mla.argtypes = [ctypes.POINTER(plx_decode_mla_args), ctypes.c_void_p]
        lib.parallax_decode_mla.restype = ctypes.c_int
        lib.parallax_decode_mla_workspace_bytes.argtypes = [ctypes.c_int32] * 2
        lib.parallax_decode_mla_workspace_bytes.restype = ctypes.c_size_t
        lib.parallax_decode_mla_num_splits.argtypes = [ctypes.c_int32] * 4
        lib.parallax_decode_mla_num_splits.restype = ctypes.c_int32
        lib.parallax_util_mfma.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p]
        lib.parallax_util_mfma.restype = ctypes.c_int
        lib.parallax_util_read_sink_slots.argtypes = []
        lib.parallax_util_read_sink_slots.restype = ctypes.c_int32
        lib.parallax_strerror.argtypes = [ctypes.c_int]
        lib.parallax_strerror.restype = ctypes.c_char_p
        lib.parallax_version.argtypes = []
        lib.parallax_version.restype = ctypes.c_int
        _lib = lib
    return _lib


def strerror(status: int) -> str:
    return load_library().parallax_strerror(int(status)).decode()


def version() -> int:
    return int(load_library().parallax_version())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return PLX_BF16
    if t.dtype == torch.float32:
        return PLX_F32
    raise TypeError("Parallax kernels take bfloat16 or float32 tensors, got %s" % t.dtype)


# (the stream's handle without the stream object around it, which takes 2.5 us to build)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_raw_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream_ptr(stream) -> int:
    if stream is None:
        if _raw_stream is not None and _raw_device is not None:
            return _raw_stream(_raw_device())
        stream = torch.cuda.current_stream()
    return int(stream.cuda_stream)


def _here() -> int:
    return _raw_device() if _raw_device is not None else torch.cuda.current_device()


def _launch_stream(where, stream) -> int:
    """_stream_ptr, of a stream of the current device only."""
    at = getattr(stream, "device_index", None)
    if at is not None and at != _here():
        raise ValueError("%s: the stream is one of device %d, which is not the current one" % (where, at))
    return _stream_ptr(stream)


def _sink_shapes(where, q, like_q, k, v):
    """Refuses tensors that do not fit each other: [B, Hq, T, d] and [B, Hkv, Tkv, d] of one type on the current device."""
    _on_current_device(where, q, k, v, *like_q)
    if q.dim() != 4 or k.dim() != 4 or v.shape != k.shape or k.shape[0] != q.shape[0] or k.shape[3] != q.shape[3]:
        raise ValueError("%s: q [B, Hq, T, d], k and v [B, Hkv, Tkv, d]" % where)
    if k.dtype != q.dtype or v.dtype != q.dtype:
        raise TypeError("%s: q, k and v have one dtype" % where)
    for t in like_q:
        if t is not None and (t.shape != q.shape or t.dtype != q.dtype or t.stride(-1) != 1):
            raise ValueError("%s: r, the outputs and their gradients have the shape and dtype of q" % where)


def _on_current_device(where, *tensors):
    """Refuses tensors (None: left out) that are not all on the current device, where the launch goes."""
    here = -1
    for t in tensors:
        if t is not None:
            at = t.get_device()
            if at < 0 or (here >= 0 and at != here):
                raise ValueError("%s needs device tensors of one device" % where)
            here = at
    if here != _here():
        raise ValueError("%s: the tensors are on device %d, which is not the current one" % (where, here))


def _bytes(t) -> int:
    return t.numel() * t.element_size()


def _ptr(t) -> int:
    return 0 if t is None else t.data_ptr()


def _other_stream(stream, device):
    """The stream that a launch goes to if it is not the current one, else None."""
    if stream is None or _stream_ptr(stream) == _stream_ptr(None):
        return None
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream.cuda_stream), device=device)


def _scratch(stream, n_floats, device):
    """fp32 scratch of a launch on `stream`, from that stream's own memory: a block of the current stream's
    may still be in use by work queued there, and may be handed out again there as soon as
    the call returns."""
    other = None if stream is None else _other_stream(stream, device)
    if other is None:
        return torch.empty(n_floats, dtype=torch.float32, device=device)
    with torch.cuda.stream(other):
        return torch.empty(n_floats, dtype=torch.float32, device=device)


def _result(stream, make, *args, **kw):
    """make(*args, **kw) (torch.empty or empty_like), a tensor that a launch on `stream` writes and the caller gets: from the launch
    stream's memory as well, and not reused there before the current stream, where the caller
    goes on, is through with it."""
    other = _other_stream(stream, kw["device"] if "device" in kw else args[0].device)
    if other is None:
        return make(*args, **kw)
    with torch.cuda.stream(other):
        t = make(*args, **kw)
    t.record_stream(torch.cuda.current_stream(t.device))
    return t


def _result_maker(stream, make):
    """`make` for the results of a launch on `stream` (itself without one: a training step of small
    shapes makes nine tensors, and is bound by the host)."""
    return make if stream is None else functools.partial(_result, stream, make)


def parallax_rope_table(n_pos, d, theta=1.0e6, device="cuda:0", stream=None):
    """(cos, sin) of pos * theta^(-2i/d): fp32 tensor [n_pos, d/2, 2] for qr_prep()."""
    table = _result_maker(stream, torch.empty)(n_pos, d // 2, 2, dtype=torch.float32, device=device)
    st = load_library().parallax_rope_table(table.data_ptr(), int(n_pos), int(d), float(theta), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_rope_table")
    return table


def qr_prep(q_gamma, r_gamma, rope_table=None, pos0=None, rope_q=True, rope_r=True, eps=1e-6):
    """Fill a plx_qr_prep (RMSNorm + RoPE on q, rho inside the attention kernels) from tensors. The
    returned struct only holds pointers: keep the tensors alive until the call has been enqueued."""
    a = plx_qr_prep()
    for g in (q_gamma, r_gamma):
        if g is not None and (g.dtype != torch.float32 or not g.is_cuda or not g.is_contiguous()):
            raise TypeError("RMSNorm weights must be contiguous fp32 device tensors")
    a.q_gamma = q_gamma.data_ptr()
    a.r_gamma = r_gamma.data_ptr() if r_gamma is not None else None
    if rope_table is not None:
        if rope_table.dtype != torch.float32 or not rope_table.is_contiguous():
            raise TypeError("rope_table must be a contiguous fp32 tensor [n_pos, d/2, 2]")
        a.rope_table, a.rope_positions = rope_table.data_ptr(), rope_table.shape[0]
        a.rope_q, a.rope_r = (1 if rope_q else 0), (1 if rope_r else 0)
    if pos0 is not None:
        if pos0.dtype != torch.int32:
            raise TypeError("pos0 must be int32")
        a.pos0 = pos0.data_ptr()
    a.eps = float(eps)
    return a


def parallax_decode_workspace_bytes(B, Hq, Hkv, Lmax, d) -> int:
    return int(load_library().parallax_decode_workspace_bytes(B, Hq, Hkv, Lmax, d))


def parallax_decode_num_splits(B, Hq, Hkv, Lmax, d, num_cus=0) -> int:
    return int(load_library().parallax_decode_num_splits(B, Hq, Hkv, Lmax, d, num_cus))


def decode_args(q, r, k, v, out, scale, seq_lens=None, use_r=True, num_splits=0, workspace=None,
                block_table=None, max_len=None, window=0, kind=plx_decode_args, tail=()):
    """Fill a plx_decode_args (or a `kind` that begins with one and goes on with the fields of `tail`) from tensors: q, r, out [B, Hq, d]; k, v [B, Hkv, Lmax, d], or,
    with block_table [B, pages per sequence] (int32), page pools [num_pages, Hkv, page_size, d]
    (max_len = largest logical length, default: pages per sequence x page_size).
    q, r, out may also be [B, Hq, Tq, d]: Tq query rows, the last Tq positions of each sequence."""
    Tq = q.shape[2] if q.dim() == 4 else 1
    B, Hq, d = q.shape[0], q.shape[1], q.shape[-1]
    num_pages, Hkv, Lmax, _ = k.shape
    paged = (0, 0, 0, 0)
    if block_table is not None:
        paged = (block_table.data_ptr(), Lmax, block_table.stride(0), num_pages)
        Lmax = _i32(max_len if max_len is not None else block_table.shape[1] * Lmax)
    return _filled(kind, q.data_ptr(), _ptr(r), k.data_ptr(), v.data_ptr(), out.data_ptr(), _ptr(seq_lens),
                   B, Hq, Hkv, Lmax, d, *k.stride()[:3], *v.stride()[:3], _f32(scale), 1 if use_r else 0, _i32(num_splits),
                   _ptr(workspace), 0 if workspace is None else _bytes(workspace), _dtype_code(q), *paged, Tq,
                   _i32(window), 0, *_NO_PREP, *tail)


def parallax_decode(q, r, k, v, scale, seq_lens=None, use_r=True, num_splits=0, workspace=None,
                    out=None, stream=None, block_table=None, max_len=None, split_counters=None,
                    window=0, prep=None, sinks=0, block_list=None):
    """Single-step Parallax decode. Allocates `out` / `workspace` with torch when not given
    (allocation only; all arithmetic is in the library). With `split_counters` (zeroed int32
    device tensor, >= B * Hkv entries) the call goes to parallax_decode_fused: one launch, the
    last split of every group to arrive merges inside the kernel. With `sinks` > 0 the first tokens stay visible
    behind the sliding window (parallax_decode_sinks; no split_counters, no prep). With `block_list` (int32 [B, Hkv, n],
    parallax_select_blocks makes one) only the keys in the listed blocks of 64 are seen (parallax_decode_blocks, bf16; neither
    window nor the others)."""
    if block_list is not None:
        if split_counters is not None or prep is not None or sinks:
            raise ValueError("a block_list goes with neither split_counters, prep nor sinks")
        return _decode_rows(q, r, k, v, scale, seq_lens, use_r, num_splits, workspace, out, stream, block_table,
                            max_len, window, 0, block_list=block_list)
    if sinks:
        if split_counters is not None or prep is not None:
            raise ValueError("sinks go with neither split_counters nor prep")
        return _decode_rows(q, r, k, v, scale, seq_lens, use_r, num_splits, workspace, out, stream, block_table,
                            max_len, window, _i32(sinks))
    if not (q.is_cuda and k.is_cuda and v.is_cuda and (r is None or r.is_cuda)):
        raise ValueError("parallax_decode needs device tensors")
    if q.stride(-1) != 1 or k.stride(-1) != 1 or v.stride(-1) != 1 or not q.is_contiguous() or (
            r is not None and not r.is_contiguous()):
        raise ValueError("q, r must be contiguous and k, v contiguous in the last dimension")
    if seq_lens is not None and seq_lens.dtype != torch.int32:
        raise TypeError("seq_lens must be int32")
    B, Hq, d = q.shape[0], q.shape[1], q.shape[-1]
    Tq = q.shape[2] if q.dim() == 4 else 1
    _, Hkv, _, _ = k.shape
    if block_table is not None:
        if block_table.dtype != torch.int32 or not block_table.is_cuda or block_table.stride(1) != 1:
            raise TypeError("block_table must be an int32 device tensor [B, pages per sequence]")
        if block_table.shape[0] != B or v.shape != k.shape:
            raise ValueError("block_table needs one row per sequence; k and v pools of one shape")
    if out is None:
        out = _result_maker(stream, torch.empty_like)(q)
    a = decode_args(q, r, k, v, out, scale, seq_lens, use_r, num_splits, workspace, block_table,
                    max_len, window)
    lib = load_library()
    if workspace is None and num_splits != 1:
        S = lib.parallax_decode_call_splits(ctypes.byref(a))  # (0: refused below)
        if S > 1:
            workspace = _scratch(stream, B * Hq * Tq * S * (2 * d + 4), q.device)
            a.workspace, a.workspace_bytes = workspace.data_ptr(), _bytes(workspace)
    if prep is not None:
        a.prep = prep
    entry = "parallax_decode"
    if split_counters is not None:
        if (split_counters.dtype != torch.int32 or not split_counters.is_cuda
                or not split_counters.is_contiguous() or split_counters.numel() < B * Hkv):
            raise TypeError("split_counters must be a contiguous int32 device tensor, >= B * Hkv")
        a.split_counters = split_counters.data_ptr()
        entry = "parallax_decode_fused"
    st = getattr(lib, entry)(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, entry)
    return out


def _decode_rows(q, r, k, v, scale, seq_lens, use_r, num_splits, workspace, out, stream, block_table, max_len, window,
                 sinks, tree_mask=None, draft_lens=None, block_list=None):
    """parallax_decode_sinks, parallax_decode_tree with a tree_mask, or parallax_decode_blocks with a block_list."""
    # (a step of one sequence is bound by the host: each property of a tensor is asked for once)
    where = "parallax_decode_sinks" if tree_mask is None else "parallax_decode_tree"
    if block_list is not None:
        where = "parallax_decode_blocks"
    _on_current_device(where, q, r, k, v, out, seq_lens, block_table, tree_mask, draft_lens, workspace, block_list)
    shape, cache, dtype = q.shape, k.shape, q.dtype
    if len(shape) not in (3, 4) or len(cache) != 4 or v.shape != cache or cache[3] != shape[-1]:
        raise ValueError("q [B, Hq, (Tq,) d], k and v of one shape [.., Hkv, .., d]")
    if use_r and r is None:
        raise ValueError("r is needed unless use_r=False")
    if (r is not None and r.shape != shape) or (out is not None and out.shape != shape):
        raise ValueError("r and out have the shape of q")
    if k.dtype != dtype or v.dtype != dtype or (r is not None and r.dtype != dtype) or (out is not None and out.dtype != dtype):
        raise TypeError("q, r, k, v and out have one dtype")
    if (k.stride(-1) != 1 or v.stride(-1) != 1 or not q.is_contiguous() or (r is not None and not r.is_contiguous())
            or (out is not None and not out.is_contiguous())):
        raise ValueError("q, r, out must be contiguous and k, v contiguous in the last dimension")
    B, Hq, d = shape[0], shape[1], shape[-1]
    Tq = shape[2] if len(shape) == 4 else 1
    for name, t in (("seq_lens", seq_lens), ("draft_lens", draft_lens)):
        if t is not None and (t.dtype != torch.int32 or t.shape != (B,) or not t.is_contiguous()):
            raise TypeError("%s must be a contiguous int32 tensor [B]" % name)
    if block_table is not None:
        if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.stride(1) != 1:
            raise TypeError("block_table must be an int32 device tensor [B, pages per sequence]")
        if block_table.shape[0] != B:
            raise ValueError("block_table needs one row per sequence")
    elif cache[0] != B:
        raise ValueError("k and v need one cache per sequence")
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    if out is None:
        out = _result_maker(stream, torch.empty_like)(q)
    given = (q, r, k, v, out, scale, seq_lens, use_r, num_splits, workspace, block_table, max_len, window)
    lib = load_library()
    if block_list is not None:
        blocks = decode_args(*given, plx_decode_blocks_args, (block_list.data_ptr(), _list_length(where, block_list, B, cache[1])))
        a = blocks.decode  # (in place)
        splits, call, head = lib.parallax_decode_blocks_call_splits, lib.parallax_decode_blocks, (ctypes.byref(blocks),)
    elif tree_mask is None:
        a = decode_args(*given)
        splits, call, head = lib.parallax_decode_sinks_call_splits, lib.parallax_decode_sinks, (ctypes.byref(a), sinks)
    else:
        words = -(-Tq // 64)
        if tree_mask.dtype != torch.int64 or not tree_mask.is_contiguous():
            raise TypeError("tree_mask must be a contiguous int64 tensor of 64-bit words")
        rows = tuple(tree_mask.shape)
        if words == 1 and rows in ((Tq,), (1, Tq), (B, Tq)):
            rows += (1,)
        if len(rows) == 2:
            rows = (1,) + rows
        if rows not in ((1, Tq, words), (B, Tq, words)):
            raise ValueError("tree_mask must be [(1 or B,) Tq, ceil(Tq/64)]")
        tree = plx_decode_tree_args()
        tree.decode, tree.tree_mask, tree.mask_batch = decode_args(*given), tree_mask.data_ptr(), rows[0]
        tree.draft_lens, tree.sinks = _ptr(draft_lens), sinks
        a = tree.decode  # (the copy inside)
        splits, call, head = lib.parallax_decode_tree_call_splits, lib.parallax_decode_tree, (ctypes.byref(tree),)
    if workspace is None and num_splits != 1:
        S = splits(*head)  # (0: refused below)
        if S > 1:
            workspace = _scratch(stream, B * Hq * Tq * S * (2 * d + 4), q.device)
            a.workspace, a.workspace_bytes = workspace.data_ptr(), _bytes(workspace)
    st = call(*head, _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)
    return out


def parallax_decode_tree(q, r, k, v, scale, tree_mask, seq_lens=None, draft_lens=None, use_r=True, num_splits=0,
                         workspace=None, out=None, stream=None, block_table=None, max_len=None, window=0, sinks=0):
    """Attention of drafted tokens that form a tree. q, r [B, Hq, Tq, d]: the nodes, whose keys and values are the last
    draft_lens[b] (default Tq) of the seq_lens[b] cached tokens. tree_mask int64 [Tq], [Tq, W], [1 or B, Tq] or
    [1 or B, Tq, W], W = ceil(Tq / 64) (tree_mask_words makes one): bit m of node t's words: it sees drafted key m. Every node sees
    the committed keys. With a window a node sees, of both, the keys inside its window and those at the first `sinks` positions, where a
    node's position is the number of its ancestors behind the committed ones. Rows from draft_lens[b] on return zeros."""
    if q.dim() != 4:
        raise ValueError("q [B, Hq, Tq, d]")
    return _decode_rows(q, r, k, v, scale, seq_lens, use_r, num_splits, workspace, out, stream, block_table, max_len,
                        window, _i32(sinks), tree_mask, draft_lens)


def tree_mask_words(parents):
    """Parents [.., Tq] (integers; the parent of node t lies before it, negative: a root) -> the mask words [.., Tq,
    ceil(Tq / 64)] (int64) of parallax_decode_tree: every node sees its ancestors and itself. Index bookkeeping only; with the parents
    on the device it waits for them at every node and cannot be captured."""
    Tq = parents.shape[-1]
    sees = torch.eye(Tq, dtype=torch.bool, device=parents.device).expand(*parents.shape, Tq).clone()
    for t in range(1, Tq):
        up = parents[..., t].long()
        if bool((up >= t).any()):
            raise ValueError("the parent of a node lies before it")
        row = sees.gather(-2, up.clamp(min=0)[..., None, None].expand(*up.shape, 1, Tq))[..., 0, :]
        sees[..., t, :] |= row & (up >= 0)[..., None]
    words = -(-Tq // 64)
    sees = torch.nn.functional.pad(sees, (0, 64 * words - Tq)).reshape(*parents.shape, words, 64)
    return (sees.long() << torch.arange(64, device=parents.device)).sum(-1)


def _list_length(where, block_list, B, Hkv):
    if block_list.dtype != torch.int32 or not block_list.is_contiguous():
        raise TypeError("%s: block_list must be a contiguous int32 tensor" % where)
    shape = block_list.shape
    if len(shape) != 3 or shape[0] != B or shape[1] != Hkv or shape[2] < 1:
        raise ValueError("%s: block_list [B, Hkv, n]" % where)
    return shape[2]


_Q4_DIMS = {144: 128, 80: 64}  # bytes of a row: its head dimension


def parallax_q4_row_bytes(d) -> int:
    """Bytes of a 4-bit row of K and V of one token and key head (0: not a head dimension that such caches have). A cache is a
    uint8 tensor [B, Hkv, capacity, row bytes], or with a block table pools [num_pages, Hkv, page_size, row bytes]; the header
    has the row."""
    return int(load_library().parallax_q4_row_bytes(_i32(d)))


def _table_fields(where, block_table, rows, pages, B):
    """(block_table, page_size, block_table_stride, num_pages) of a call over B sequences, and their capacity."""
    if block_table is None:
        if pages != B:
            raise ValueError("%s: a cache has one slot per sequence" % where)
        return (0, 0, 0, 0), rows
    if block_table.dtype != torch.int32 or block_table.dim() != 2 or block_table.stride(1) != 1:
        raise TypeError("%s: block_table must be an int32 device tensor [B, pages per sequence]" % where)
    if block_table.shape[0] != B:
        raise ValueError("%s: block_table needs one row per sequence" % where)
    width = block_table.shape[1]
    return (block_table.data_ptr(), rows, block_table.stride(0) if B > 1 else width, pages), min(width * rows, 0x7fffffff)


def _lens(where, name, t, B):
    if t is None:
        return 0
    if t.dtype != torch.int32 or t.shape != (B,) or not t.is_contiguous():
        raise TypeError("%s: %s must be a contiguous int32 tensor [B]" % (where, name))
    return t.data_ptr()


def _q4_fields(where, cache, block_table, B, d=None, max_len=None):
    """The fields of a plx_q4_cache."""
    shape = cache.shape
    if cache.dtype != torch.uint8 or len(shape) != 4 or cache.stride(3) != 1 or shape[3] not in _Q4_DIMS:
        raise TypeError("%s: a 4-bit cache is a uint8 tensor [.., Hkv, .., row bytes], contiguous in the last dimension" % where)
    if d is not None and _Q4_DIMS[shape[3]] != d:
        raise ValueError("%s: the cache has rows of d = %d" % (where, _Q4_DIMS[shape[3]]))
    table, capacity = _table_fields(where, block_table, shape[2], shape[0], B)
    if max_len is not None:
        capacity = min(_i32(max_len), capacity)
    return (cache.data_ptr(), *cache.stride()[:3], *table, B, shape[1], capacity, _Q4_DIMS[shape[3]])


def _q4_rows(where, call, cache, k, v, start, counts, block_table, stream):
    if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype or k.stride(3) != 1 or v.stride(3) != 1:
        raise ValueError("%s: k and v [B, Hkv, T, d] of one dtype, contiguous in the last dimension" % where)
    B, Hkv, T, d = k.shape
    if cache.dim() != 4 or cache.shape[1] != Hkv:
        raise ValueError("%s: the cache has as many heads as k and v" % where)
    a = _filled(plx_q4_rows_args, *_q4_fields(where, cache, block_table, B, d), k.data_ptr(), v.data_ptr(), *k.stride()[:3],
                *v.stride()[:3], _lens(where, "start", start, B), _lens(where, "counts", counts, B), T, _dtype_code(k))
    if T == 0:
        return
    st = call(ctypes.byref(a), _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)


def parallax_cache_write_q4(k, v, cache, start=None, counts=None, block_table=None, stream=None):
    """Rows of K and V [B, Hkv, T, d] (bf16 or fp32) into a 4-bit cache: row t of sequence b becomes its token start[b] + t
    (default 0); rows from counts[b] on are passed over. Tokens outside the cache, and those without a page, are not written."""
    where = "parallax_cache_write_q4"
    _on_current_device(where, k, v, cache, start, counts, block_table)
    _q4_rows(where, load_library().parallax_cache_write_q4, cache, k, v, start, counts, block_table, stream)


def parallax_cache_read_q4(cache, d, T, start=None, seq_lens=None, dtype=torch.bfloat16, block_table=None, out=None,
                           stream=None):
    """The values that T tokens of every sequence stand for, from start[b] (default 0) on, as k, v [B, Hkv, T, d] in `dtype` (bf16: exact):
    what parallax_prefill takes as the keys in front of the next chunk. Tokens from seq_lens[b] on, outside the cache or without a page:
    zeros. out: (k, v) to write."""
    where = "parallax_cache_read_q4"
    _on_current_device(where, cache, start, seq_lens, block_table, *(out or ()))
    B = cache.shape[0] if block_table is None else block_table.shape[0]
    if out is None:
        make = _result_maker(stream, torch.empty)
        out = [make((B, cache.shape[1], T, d), dtype=dtype, device=cache.device) for _ in range(2)]
    k, v = out
    if tuple(k.shape) != (B, cache.shape[1], T, d) or any(s == 0 and n > 1 for t in (k, v) for s, n in zip(t.stride(), t.shape)):
        raise ValueError("%s: out is (k, v), each [B, Hkv, T, d] with a place for every value" % where)
    _q4_rows(where, load_library().parallax_cache_read_q4, cache, k, v, start, seq_lens, block_table, stream)
    return k, v


def parallax_decode_q4(q, r, cache, scale, seq_lens=None, use_r=True, num_splits=0, workspace=None, out=None, stream=None,
                       block_table=None, max_len=None, window=0, sinks=0, block_list=None):
    """parallax_decode over a cache held in 4 bits: q, r [B, Hq, (Tq,) d] bf16, at most 16 rows x heads of a group; window and
    sinks as parallax_decode, or a block_list."""
    where = "parallax_decode_q4"
    _on_current_device(where, q, r, cache, out, seq_lens, block_table, block_list, workspace)
    shape = q.shape
    if len(shape) not in (3, 4):
        raise ValueError("q [B, Hq, (Tq,) d]")
    if use_r and r is None:
        raise ValueError("r is needed unless use_r=False")
    for t in (q, r, out):
        if t is not None and (t.shape != shape or t.dtype != torch.bfloat16 or not t.is_contiguous()):
            raise ValueError("q, r and out are contiguous bf16 tensors of one shape")
    B, Hq, d = shape[0], shape[1], shape[-1]
    Tq = shape[2] if len(shape) == 4 else 1
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    fields = _q4_fields(where, cache, block_table, B, d, max_len)
    Hkv = fields[9]
    n_list = 0 if block_list is None else _list_length(where, block_list, B, Hkv)
    if out is None:
        out = _result_maker(stream, torch.empty_like)(q)
    # (in one go: see _PACK)
    a = _filled(plx_decode_q4_args, q.data_ptr(), _ptr(r), 0, 0, out.data_ptr(), _lens(where, "seq_lens", seq_lens, B), B, Hq, Hkv,
                fields[10], d, 0, 0, 0, 0, 0, 0, _f32(scale), 1 if use_r else 0, _i32(num_splits), _ptr(workspace),
                0 if workspace is None else _bytes(workspace), PLX_BF16, 0, 0, 0, 0, Tq, _i32(window), 0, *_NO_PREP,
                *fields, _i32(sinks), n_list, _ptr(block_list))
    lib = load_library()
    if workspace is None and num_splits != 1:
        S = lib.parallax_decode_q4_call_splits(ctypes.byref(a))  # (0: refused below)
        if S > 1:
            workspace = _scratch(stream, B * Hq * Tq * S * (2 * d + 4), q.device)
            a.decode.workspace, a.decode.workspace_bytes = workspace.data_ptr(), _bytes(workspace)
    st = lib.parallax_decode_q4(ctypes.byref(a), _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)
    return out


def parallax_cache_bounds(k, bounds, seq_lens=None, from_lens=None, max_new=0, block_table=None, stream=None, max_len=None):
    """The smallest and largest key of every block of 64 tokens, by dimension, into bounds [B, Hkv, n_blocks, 2, d] (bf16), which is
    returned. k: the bf16 keys [B, Hkv, capacity, d] or pools of a block_table, or a 4-bit cache. from_lens: the tokens in
    front of these are the same as when the bounds were last brought up to date; only blocks from there on are looked at. max_new: no
    sequence holds more tokens behind its from_lens (0: not known). max_len: no sequence of a block_table is longer (default: what its pages
    hold, as far as that only rounds up to whole pages); bounds with fewer blocks than that takes are refused."""
    where = "parallax_cache_bounds"
    _on_current_device(where, k, bounds, seq_lens, from_lens, block_table)
    if k.dim() != 4 or bounds.dim() != 5:
        raise ValueError("%s: keys [.., Hkv, .., d], bounds [B, Hkv, n_blocks, 2, d]" % where)
    B, Hkv, n_blocks, two, d = bounds.shape
    if bounds.dtype != torch.bfloat16 or not bounds.is_contiguous() or two != 2 or k.shape[1] != Hkv:
        raise ValueError("%s: bounds is a contiguous bf16 tensor [B, Hkv, n_blocks, 2, d]" % where)
    most = min(64 * n_blocks, 0x7fffffff)
    tokens = k.shape[2]  # at least
    if max_len is not None:
        tokens = _i32(max_len)
        if tokens < 1:
            raise ValueError("%s: max_len must be at least 1" % where)
        if block_table is None and tokens > k.shape[2]:
            raise ValueError("%s: the cache holds %d tokens" % (where, k.shape[2]))
    elif block_table is not None:
        tokens = (block_table.shape[-1] - 1) * k.shape[2] + 1
    if tokens > most:
        raise ValueError("%s: bounds for %d blocks are too few for %d tokens%s" %
                         (where, n_blocks, tokens, "" if block_table is None or max_len is not None else " (or give max_len)"))
    if max_len is not None:
        most = tokens
    lens = _lens(where, "seq_lens", seq_lens, B), _lens(where, "from_lens", from_lens, B)
    tail = (bounds.data_ptr(), n_blocks, _i32(max_new), *lens)
    if k.dtype == torch.uint8:
        cache = _filled(plx_q4_cache, *_q4_fields(where, k, block_table, B, d, most))
        a = _filled(plx_cache_bounds_args, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, ctypes.addressof(cache), *tail)
    else:
        if k.dtype != torch.bfloat16 or k.stride(3) != 1 or k.shape[3] != d:
            raise TypeError("%s: keys are bf16 [.., Hkv, .., d], contiguous in the last dimension, or a 4-bit cache" % where)
        table, capacity = _table_fields(where, block_table, k.shape[2], k.shape[0], B)
        a = _filled(plx_cache_bounds_args, k.data_ptr(), *k.stride()[:3], *table, B, Hkv, min(capacity, most), d, 0, *tail)
    st = load_library().parallax_cache_bounds(ctypes.byref(a), _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)
    return bounds


def parallax_select_blocks(q, bounds, seq_lens, keep, first=1, recent=2, out=None, workspace=None, stream=None):
    """The blocks that a step with queries q [B, Hq, (Tq,) d] reads: int32 [B, Hkv, keep], ascending, -1 behind the last: the
    `first` ones, the `recent` last ones, and of the others those with the highest bound on a product with one of the queries
    (of the rows and heads that share a key head; of equal ones the lower number). A sequence has no more blocks than bounds: of a longer one
    the `recent` ones are the last that have any."""
    where = "parallax_select_blocks"
    _on_current_device(where, q, bounds, seq_lens, out, workspace)
    shape = q.shape
    if len(shape) not in (3, 4) or q.dtype != torch.bfloat16 or not q.is_contiguous():
        raise ValueError("%s: q is a contiguous bf16 tensor [B, Hq, (Tq,) d]" % where)
    B, Hq, d = shape[0], shape[1], shape[-1]
    Tq = shape[2] if len(shape) == 4 else 1
    held = bounds.shape
    if len(held) != 5 or bounds.dtype != torch.bfloat16 or not bounds.is_contiguous() or held[0] != B or held[3] != 2 or held[4] != d:
        raise ValueError("%s: bounds is a contiguous bf16 tensor [B, Hkv, n_blocks, 2, d]" % where)
    Hkv, n_blocks = held[1], held[2]
    lens, keep = _lens(where, "seq_lens", seq_lens, B), _i32(keep)
    if out is None:
        out = _result_maker(stream, torch.empty)((B, Hkv, max(keep, 0)), dtype=torch.int32, device=q.device)
    elif _list_length(where, out, B, Hkv) != keep:
        raise ValueError("%s: out [B, Hkv, keep]" % where)
    lib = load_library()
    if workspace is None:
        workspace = _scratch(stream, lib.parallax_select_blocks_workspace_bytes(B, Hkv, n_blocks) // 4, q.device)
    elif not workspace.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    a = _filled(plx_select_blocks_args, q.data_ptr(), bounds.data_ptr(), lens, out.data_ptr(), B, Hq, Hkv, Tq, d, n_blocks, keep,
                _i32(first), _i32(recent), workspace.data_ptr(), _bytes(workspace))
    st = lib.parallax_select_blocks(ctypes.byref(a), _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)
    return out


def parallax_decode_static_scratch_bytes() -> int:
    return int(load_library().parallax_decode_static_scratch_bytes())


def parallax_decode_static(q, r, k, v, scale, out, seq_lens=None, use_r=True, num_splits=0,
                           stream=None, block_table=None, max_len=None, window=0):
    """parallax_decode with the split records in the library's own fixed scratch: nothing is
    allocated here or in the library; `out` is the caller's."""
    a = decode_args(q, r, k, v, out, scale, seq_lens, use_r, num_splits, None, block_table, max_len,
                    window)
    st = load_library().parallax_decode_static(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_decode_static")
    return out


def parallax_decode_fused(q, r, k, v, scale, split_counters, **kw):
    """parallax_decode with the merge inside the split kernel; see parallax_decode."""
    return parallax_decode(q, r, k, v, scale, split_counters=split_counters, **kw)


def parallax_decode_partials(q, r, k, v, scale, num_splits, workspace, seq_lens=None, use_r=True,
                             stream=None):
    """Split kernel only: fills `workspace` with the (m, d1, d2, pad, O1, O2) records."""
    a = decode_args(q, r, k, v, q, scale, seq_lens, use_r, num_splits, workspace)
    a.o = None
    st = load_library().parallax_decode_partials(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_decode_partials")
    return workspace


def parallax_decode_combine(workspace, out, Hkv, num_splits, stream=None):
    """Merge kernel only: `workspace` holds num_splits records per (b, hq); writes out [B, Hq, d]."""
    B, Hq, d = out.shape
    a = plx_decode_args()
    a.o = out.data_ptr()
    a.B, a.Hq, a.Hkv, a.Lmax, a.d = B, Hq, Hkv, 1, d
    a.num_splits = int(num_splits)
    a.workspace = workspace.data_ptr()
    a.workspace_bytes = workspace.numel() * workspace.element_size()
    a.dtype = _dtype_code(out)
    st = load_library().parallax_decode_combine(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_decode_combine")
    return out


def prefill_args(q, r, k, v, out, scale, causal=True, use_r=True, window=0):
    """Fill a plx_prefill_args from tensors: q, r, out [B, Hq, T, d]; k, v [B, Hkv, Tkv, d]."""
    B, Hq, T, d = q.shape
    Hkv, Tkv = k.shape[1], k.shape[2]
    q_stride = q.stride()[:3]
    return _filled(plx_prefill_args, q.data_ptr(), _ptr(r), k.data_ptr(), v.data_ptr(), out.data_ptr(), B, Hq, Hkv, T, d,
                   *q_stride, *(r.stride()[:3] if r is not None else q_stride), *k.stride()[:3], *v.stride()[:3],
                   *out.stride()[:3], _f32(scale), 1 if causal else 0, 1 if use_r else 0, _dtype_code(q), Tkv, _i32(window),
                   0, 0, 0, 0, 0, 0, *_NO_PREP)


BLOCK_ROWS, BLOCK_KEYS = 128, 64  # the block-sparse granularity: the prefill kernel's tiles


def block_mask_lists(block_mask):
    """Block mask [(B,) (Hq,) ceil(T/128), ceil(Tkv/64)] (bool, device) -> (row_ptr, tile_idx,
    sparse_batch, sparse_heads) for plx_prefill_args: per row block the ascending indices of its
    key tiles. Index bookkeeping only."""
    m = block_mask.to(torch.bool)
    while m.dim() < 4:
        m = m.unsqueeze(0)
    Bs, Hs, nrb, nkt = m.shape
    flat = m.reshape(-1, nkt)
    counts = flat.sum(dim=1)
    row_ptr = torch.zeros(flat.shape[0] + 1, dtype=torch.int32, device=m.device)
    row_ptr[1:] = torch.cumsum(counts, 0).to(torch.int32)
    tile_idx = torch.nonzero(flat)[:, 1].to(torch.int32).contiguous()  # row-major: ascending per row
    if tile_idx.numel() == 0:
        tile_idx = torch.zeros(1, dtype=torch.int32, device=m.device)
    return row_ptr, tile_idx, Bs, Hs


def block_mask_column_lists(block_mask):
    """The same cells by columns, for plx_prefill_bwd_args: per key block of 128 keys (two key
    tiles) the ascending row blocks that list one of its tiles, each entry 4 * row block + flags
    (flag bit t: key tile 2 * cb + t is listed). Returns (col_ptr, col_idx). Index bookkeeping only."""
    m = block_mask.to(torch.bool)
    while m.dim() < 4:
        m = m.unsqueeze(0)
    Bs, Hs, nrb, nkt = m.shape
    if nkt % 2:
        m = torch.cat([m, torch.zeros(Bs, Hs, nrb, 1, dtype=torch.bool, device=m.device)], dim=-1)
    pair = m.reshape(Bs, Hs, nrb, -1, 2)                      # [.., rb, cb, t]
    flags = pair[..., 0].to(torch.int32) + 2 * pair[..., 1].to(torch.int32)
    by_col = flags.transpose(-1, -2).reshape(-1, nrb)         # one line per (sb, sh, cb)
    hit = by_col > 0
    col_ptr = torch.zeros(by_col.shape[0] + 1, dtype=torch.int32, device=m.device)
    col_ptr[1:] = torch.cumsum(hit.sum(dim=1), 0).to(torch.int32)
    where = torch.nonzero(hit)                                # row-major: ascending row blocks per line
    col_idx = (4 * where[:, 1].to(torch.int32) + by_col[hit]).to(torch.int32).contiguous()
    if col_idx.numel() == 0:
        col_idx = torch.zeros(1, dtype=torch.int32, device=m.device)
    return col_ptr, col_idx


# What parallax_block_lists takes: entries in 32 bits, lines (row blocks + key blocks of all lists)
_MAX_LIST_CELLS, _MAX_LIST_LINES = 0x7fffffff, 1 << 25


def attach_block_lists(a, block_mask, device, stream=None, columns=False):
    """Build the lists of a block mask on the device (current stream) and point the prefill (columns:
    backward) arguments `a` at them, for a launch on `stream`. Returns the buffer that holds them
    (several tensors for a mask beyond what parallax_block_lists takes): keep it until the call has
    been enqueued."""
    m = block_mask
    if m.dtype != torch.bool or m.device != device:
        m = m.to(device=device, dtype=torch.bool)
    Bs, Hs, nrb, nkt = (1,) * (4 - m.dim()) + tuple(m.shape)
    rows, cols = Bs * Hs * nrb, Bs * Hs * ((nkt + 1) // 2)
    col_ptr = col_idx = 0
    if rows * nkt > _MAX_LIST_CELLS or rows + cols > _MAX_LIST_LINES:
        held = list(block_mask_lists(m)[:2])
        if columns:
            held += block_mask_column_lists(m)
        row_ptr, tile_idx, col_ptr, col_idx = ([t.data_ptr() for t in held] + [0, 0])[:4]
    else:
        m = m.contiguous()
        if not columns:
            cols = 0
        # [row_ptr | col_ptr | counts | tile_idx | col_idx]
        counts = rows + 1 + (cols + 1 if columns else 0)
        tiles = counts + rows + cols
        held = [torch.empty(tiles + rows * nkt + cols * nrb, dtype=torch.int32, device=device)]
        row_ptr = held[0].data_ptr()
        tile_idx = row_ptr + 4 * tiles
        if columns:
            col_ptr, col_idx = row_ptr + 4 * (rows + 1), tile_idx + 4 * rows * nkt
        la = _filled(plx_block_list_args, m.data_ptr(), Bs * Hs, nrb, nkt, row_ptr + 4 * counts, row_ptr, tile_idx, col_ptr, col_idx)
        st = load_library().parallax_block_lists(ctypes.byref(la), _stream_ptr(None))
        if st != PLX_OK:
            raise ParallaxError(st, "parallax_block_lists")
    if columns:
        _ALL_LISTS.pack_into(a, plx_prefill_bwd_args.sparse_row_ptr.offset, row_ptr, tile_idx, col_ptr, col_idx, Bs, Hs)
    else:
        _ROW_LISTS.pack_into(a, type(a).sparse_row_ptr.offset, row_ptr, tile_idx, Bs, Hs)
    other = _other_stream(stream, device)
    if other is not None:  # read there: after the lists are built, and not reused here before
        for t in held:
            t.record_stream(other)
        other.wait_stream(torch.cuda.current_stream())
    return held[0] if len(held) == 1 else held


def parallax_prefill(q, r, k, v, scale, causal=True, use_r=True, out=None, stream=None, window=0,
                     save_for_backward=False, block_mask=None, prep=None, sinks=0):
    """Parallax prefill forward over T query rows and Tkv keys (causal: the rows are the last
    T positions of the Tkv-long sequence). With save_for_backward the kernel also writes the row
    cache of the backward pass and (out, vbar, row_stats) is returned. With sinks > 0 the first tokens stay visible
    behind the sliding window (no block_mask, no prep)."""
    if sinks:
        if block_mask is not None or prep is not None:
            raise ValueError("sinks go with neither block_mask nor prep")
        _sink_shapes("parallax_prefill_sinks", q, (r, out), k, v)
        if use_r and r is None:
            raise ValueError("r is needed unless use_r=False")
    for t in (q, k, v) + ((r,) if r is not None else ()):
        if not t.is_cuda:
            raise ValueError("parallax_prefill needs device tensors")
        if t.stride(-1) != 1:
            raise ValueError("the last dimension must be contiguous")
    if v.shape[2] != k.shape[2]:
        raise ValueError("k and v must hold the same number of keys")
    if out is None:
        out = _result_maker(stream, torch.empty_like)(q)
    a = prefill_args(q, r, k, v, out, scale, causal, use_r, window)
    if block_mask is not None:
        nrb, nkt = -(-q.shape[2] // BLOCK_ROWS), -(-k.shape[2] // BLOCK_KEYS)
        if tuple(block_mask.shape[-2:]) != (nrb, nkt):
            raise ValueError("block_mask must end in [ceil(T/128), ceil(Tkv/64)] = [%d, %d]" % (nrb, nkt))
        lists = attach_block_lists(a, block_mask, q.device, stream)  # alive until the launch below
    if prep is not None:
        a.prep = prep
    if save_for_backward:
        vbar = _result_maker(stream, torch.empty_like)(out)
        if vbar.stride() != out.stride():  # (out has gaps: the kernel writes vbar with out's strides)
            vbar = _result_maker(stream, torch.empty_strided)(out.shape, out.stride(), dtype=out.dtype, device=out.device)
        B, Hq, T, _ = q.shape
        row_stats = _result_maker(stream, torch.empty)(B, Hq, T, 2, dtype=torch.float32, device=q.device)
        _ROW_CACHE.pack_into(a, plx_prefill_args.vbar.offset, vbar.data_ptr(), row_stats.data_ptr())
    lib, where = load_library(), _launch_stream("parallax_prefill_sinks", stream) if sinks else _stream_ptr(stream)
    split_bytes = 0 if sinks else lib.parallax_prefill_workspace_bytes(ctypes.byref(a))
    if sinks:
        st = lib.parallax_prefill_sinks(ctypes.byref(a), _i32(sinks), where)
    elif split_bytes:  # few row blocks, many keys: split over key ranges
        workspace = _scratch(stream, split_bytes // 4, q.device)
        st = lib.parallax_prefill_split(ctypes.byref(a), workspace.data_ptr(), split_bytes, where)
    else:
        st = lib.parallax_prefill(ctypes.byref(a), where)
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_prefill_sinks" if sinks else "parallax_prefill")
    return (out, vbar, row_stats) if save_for_backward else out


def parallax_prefill_backward_workspace_bytes(B, Hq, T) -> int:
    return int(load_library().parallax_prefill_backward_workspace_bytes(B, Hq, T))


def prefill_bwd_args(q, r, k, v, o, vbar, row_stats, d_o, dq, dr, dk, dv, scale, causal, workspace, window=0):
    """Fill a plx_prefill_bwd_args: [B, H, T, d] tensors (views with any batch / head / row strides,
    last dimension contiguous); row_stats and the workspace dense."""
    strides, ok = [], row_stats.is_cuda and workspace.is_cuda and row_stats.stride(-1) == workspace.stride(-1) == 1
    for t in (q, r, k, v, o, vbar, d_o, dq, dr, dk, dv):
        at = t.stride()
        ok = ok and t.is_cuda and at[-1] == 1
        strides += at[:3]
    if not ok:
        raise ValueError("parallax_prefill_backward needs device tensors with a contiguous last dimension")
    if not row_stats.is_contiguous() or not workspace.is_contiguous():
        raise ValueError("row_stats and the workspace must be contiguous")
    B, Hq, T, d = q.shape
    ptrs = [t.data_ptr() for t in (q, r, k, v, o, vbar, row_stats, d_o, dq, dr, dk, dv)]
    return _filled(plx_prefill_bwd_args, *ptrs, B, Hq, k.shape[1], T, k.shape[2], d, _f32(scale), 1 if causal else 0,
                   _dtype_code(q), _i32(window), workspace.data_ptr(), _bytes(workspace), *strides, 0, 0, 0, 0, 0, 0)


def parallax_prefill_backward(q, r, k, v, o, vbar, row_stats, d_o, scale, causal=True, stream=None,
                              workspace=None, window=0, block_mask=None, sinks=0):
    """Gradients (dq, dr, dk, dv) of parallax_prefill for the upstream gradient d_o, from the
    forward's output and row cache (save_for_backward=True, same causal / window / block_mask / sinks)."""
    if sinks:
        if block_mask is not None:
            raise ValueError("sinks do not go with a block_mask")
        _sink_shapes("parallax_prefill_backward_sinks", q, (r, o, vbar, d_o), k, v)
        if row_stats.dtype != torch.float32 or row_stats.shape != (*q.shape[:3], 2) or row_stats.device != q.device:
            raise ValueError("row_stats is the float32 [B, Hq, T, 2] of the forward")
    like = _result_maker(stream, torch.empty_like)
    dq, dr, dk, dv = like(q), like(q), like(k), like(k)
    own_scratch = workspace is None
    if own_scratch and not sinks:
        workspace = _scratch(stream, q.shape[0] * q.shape[1] * q.shape[2] * 4, q.device)
    # (with sinks the library says how much; row_stats in the place of the workspace until then)
    a = prefill_bwd_args(q, r, k, v, o, vbar, row_stats, d_o, dq, dr, dk, dv, scale, causal,
                         row_stats if workspace is None else workspace, window)
    if sinks:
        lib = load_library()
        if own_scratch:
            need = lib.parallax_prefill_backward_sinks_workspace_bytes(ctypes.byref(a), _i32(sinks))  # (0: refused below)
            workspace = _scratch(stream, max(need // 4, 2 * row_stats.numel()), q.device)
            a.workspace, a.workspace_bytes = workspace.data_ptr(), _bytes(workspace)
        st = lib.parallax_prefill_backward_sinks(ctypes.byref(a), _i32(sinks),
                                                 _launch_stream("parallax_prefill_backward_sinks", stream))
        if st != PLX_OK:
            raise ParallaxError(st, "parallax_prefill_backward_sinks")
        return dq, dr, dk, dv
    if block_mask is not None:
        nrb, nkt = -(-q.shape[2] // BLOCK_ROWS), -(-k.shape[2] // BLOCK_KEYS)
        if tuple(block_mask.shape[-2:]) != (nrb, nkt):
            raise ValueError("block_mask must end in [ceil(T/128), ceil(Tkv/64)] = [%d, %d]" % (nrb, nkt))
        lists = attach_block_lists(a, block_mask, q.device, stream, columns=True)  # alive until the launch below
    st = load_library().parallax_prefill_backward(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_prefill_backward")
    return dq, dr, dk, dv


def norm_rope_args(tensors, pos0=None, eps=1e-6, theta=1.0e6, rope_table=None):
    """Fill a plx_norm_rope_args. tensors: up to three (x, gamma, rope, out) with x, out
    [B, H, T, d] contiguous (out may be x) and gamma [d] fp32."""
    B, _, T, d = tensors[0][0].shape
    flat = []
    for x, gamma, use_rope, out in tensors:
        if not (x.is_cuda and x.is_contiguous() and out.is_contiguous() and gamma.dtype == torch.float32):
            raise ValueError("parallax_norm_rope needs contiguous device tensors and fp32 weights")
        if x.shape[0] != B or x.shape[2] != T or x.shape[3] != d or out.shape != x.shape:
            raise ValueError("the tensors of one call share B, T and d")
        flat += (x.data_ptr(), out.data_ptr(), gamma.data_ptr(), x.shape[1], 1 if use_rope else 0)
    if len(tensors) > 3:
        raise IndexError("at most three tensors per call")
    flat += (0,) * (15 - len(flat))
    table, n_pos = 0, 0
    if rope_table is not None:  # [n_pos, d / 2, 2] fp32 from parallax_rope_table (same d, theta)
        if rope_table.dtype != torch.float32 or not rope_table.is_contiguous() or rope_table.shape[1] != d // 2:
            raise ValueError("rope_table must be the contiguous fp32 [n_pos, d/2, 2] table of this d")
        table, n_pos = rope_table.data_ptr(), rope_table.shape[0]
    return _filled(plx_norm_rope_args, *flat, len(tensors), B, T, d, _ptr(pos0), _f32(eps), _f32(theta),
                   _dtype_code(tensors[0][0]), table, n_pos)


def parallax_norm_rope(tensors, pos0=None, eps=1e-6, theta=1.0e6, stream=None, inplace=False, rope_table=None):
    """RMSNorm + RoPE on up to three tensors in one launch. tensors: list of (x, gamma, rope);
    returns the list of results (the inputs themselves with inplace=True)."""
    if pos0 is not None and pos0.dtype != torch.int32:
        raise TypeError("pos0 must be int32")
    like = _result_maker(stream, torch.empty_like)
    full = [(x, g, rp, x if inplace else like(x)) for (x, g, rp) in tensors]
    a = norm_rope_args(full, pos0, eps, theta, rope_table)
    st = load_library().parallax_norm_rope(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_norm_rope")
    return [t[3] for t in full]


def parallax_decode_mla_workspace_bytes(B, Hq) -> int:
    return int(load_library().parallax_decode_mla_workspace_bytes(B, Hq))


def parallax_decode_mla_num_splits(B, Hq, Lmax, num_cus=0) -> int:
    return int(load_library().parallax_decode_mla_num_splits(B, Hq, Lmax, num_cus))


def decode_mla_args(q, r, ckv, out, scale, seq_lens=None, num_splits=0, workspace=None, d_latent=512,
                    block_table=None, max_len=None, window=0):
    """Fill a plx_decode_mla_args: q, r [B, Hq, dk] and out [B, Hq, d_latent] contiguous (or, with
    several query rows per head at the last positions of the sequence, [B, Hq, Tq, dk] and
    [B, Hq, Tq, d_latent]), ckv [B, L, dk] with any batch / token strides -- or, with an int32
    block_table [B, pages], a page pool [num_pages, page_size, dk] (max_len = capacity in tokens,
    default pages * page_size)."""
    for t in (q, r, out):
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError("parallax_decode_mla needs contiguous device tensors for q, r and out")
    if not ckv.is_cuda or ckv.stride(-1) != 1:
        raise ValueError("the last dimension of the cache must be contiguous")
    paged, Lmax = (0, 0, 0, 0), ckv.shape[1]
    if block_table is not None:
        if block_table.dtype != torch.int32 or not block_table.is_cuda or block_table.stride(-1) != 1:
            raise ValueError("block_table must be a device int32 tensor with a contiguous last dimension")
        paged = (block_table.data_ptr(), ckv.shape[1], ckv.shape[0], block_table.stride(0))
        Lmax = _i32(max_len if max_len is not None else block_table.shape[1] * ckv.shape[1])
    return _filled(plx_decode_mla_args, q.data_ptr(), r.data_ptr(), ckv.data_ptr(), out.data_ptr(), _ptr(seq_lens),
                   q.shape[0], q.shape[1], Lmax, d_latent, q.shape[-1] - d_latent, _i32(num_splits), ckv.stride(0),
                   ckv.stride(1), _f32(scale), _dtype_code(q), _ptr(workspace), 0 if workspace is None else _bytes(workspace), *paged,
                   q.shape[2] if q.dim() == 4 else 1, _i32(window))


def parallax_decode_mla(q, r, ckv, scale, seq_lens=None, num_splits=0, out=None, workspace=None,
                        stream=None, d_latent=512, block_table=None, max_len=None, window=0):
    """Parallax attention over an MLA-style latent cache: key = the whole cached row, value = its
    first d_latent numbers, shared by all heads. q, r [B, Hq, dk] (one decode row) or
    [B, Hq, Tq, dk] (rows at the last Tq positions, causal among themselves: a chunked decode
    step, or the prefill over the latent cache with Tq = prompt length); window > 0 = sliding."""
    if out is None:
        out = _result_maker(stream, torch.empty)(q.shape[:-1] + (d_latent,), dtype=q.dtype, device=q.device)
    n_cols = q.shape[1] * (q.shape[2] if q.dim() == 4 else 1)
    if workspace is None and num_splits != 1:
        lmax = ckv.shape[1] if block_table is None else (
            int(max_len) if max_len is not None else block_table.shape[1] * ckv.shape[1])
        S = num_splits or parallax_decode_mla_num_splits(q.shape[0], n_cols, lmax)
        if S > 1:
            workspace = _scratch(stream, q.shape[0] * n_cols * S * (2 * d_latent + 4), q.device)
    a = decode_mla_args(q, r, ckv, out, scale, seq_lens, num_splits, workspace, d_latent, block_table, max_len,
                        window)
    st = load_library().parallax_decode_mla(ctypes.byref(a), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_decode_mla")
    return out


def _int_list(where, name, t, n=None, device=None):
    at = t.get_device()
    if at < 0 or t.dtype != torch.int32 or not t.is_contiguous():
        raise TypeError("%s: %s must be a contiguous int32 device tensor" % (where, name))
    if n is not None and t.numel() != n:
        raise ValueError("%s: %s must have %d entries" % (where, name, n))
    if device is not None and at != device:
        raise ValueError("%s: %s is on another device" % (where, name))
    return t.data_ptr()


def _table_device(where, pages):
    """The device of a PageTable, which is the one that the launch goes to."""
    if pages._device != _here():
        raise ValueError("%s: the table is on device %d, which is not the current one" % (where, pages._device))
    return pages._device


class PageTable:
    """Which pages the sequences of a paged cache hold, on the device: block_table [sequences, pages per sequence], seq_lens
    [sequences], page_refs [num_pages], free_pages [num_pages], free_count [1], all int32 (see plx_page_table). The
    tensors are the caller's and are what parallax_decode and the others take as block_table and seq_lens; `empty` makes
    those of a cache nobody uses yet."""

    __slots__ = ("block_table", "seq_lens", "page_refs", "free_pages", "free_count", "page_size", "_args", "_device")

    def __init__(self, block_table, seq_lens, page_refs, free_pages, free_count, page_size):
        if block_table.dtype != torch.int32 or not block_table.is_cuda or block_table.dim() != 2 or block_table.stride(1) != 1:
            raise TypeError("block_table must be an int32 device tensor [sequences, pages per sequence]")
        device, (sequences, width), pages = block_table.get_device(), block_table.shape, page_refs.numel()
        ptrs = [_int_list("PageTable", name, t, n, device) for name, t, n in (
            ("seq_lens", seq_lens, sequences), ("page_refs", page_refs, pages), ("free_pages", free_pages, pages),
            ("free_count", free_count, 1))]
        self.block_table, self.seq_lens, self.page_refs = block_table, seq_lens, page_refs
        self.free_pages, self.free_count, self.page_size, self._device = free_pages, free_count, int(page_size), device
        self._args = _filled(plx_page_table, block_table.data_ptr(), *ptrs, sequences, width,
                             block_table.stride(0) if sequences > 1 else width, pages, _i32(page_size))

    @classmethod
    def empty(cls, sequences, pages_per_sequence, num_pages, page_size, device="cuda:0"):
        opts = dict(dtype=torch.int32, device=device)
        return cls(torch.full((sequences, pages_per_sequence), -1, **opts), torch.zeros(sequences, **opts),
                   torch.zeros(num_pages, **opts), torch.arange(num_pages - 1, -1, -1, **opts),
                   torch.full((1,), num_pages, **opts), page_size)


def _pools(where, k, v):
    """The fields of a plx_cache_pools: [pages, heads, rows, d], or [pages, rows, d] for one head; pools of 4-bit rows (uint8, no v)
    as pools of bf16 rows of half as many numbers."""
    if k.dtype == torch.uint8 and v is None:
        k = k.view(torch.bfloat16)
    if k.dim() == 3:
        k = k.unsqueeze(1)
    _on_current_device(where, k, v)
    if k.dim() != 4 or k.stride(-1) != 1:
        raise ValueError("%s needs device pools [num_pages, (heads,) page_size, d], contiguous in the last dimension" % where)
    vs = (0, 0, 0)
    if v is not None:
        if v.dim() == 3:
            v = v.unsqueeze(1)
        if v.shape != k.shape or v.dtype != k.dtype or v.stride(-1) != 1:
            raise ValueError("%s: k and v are pools of one shape and type" % where)
        vs = v.stride()[:3]
    pages, heads, rows, d = k.shape
    return (k.data_ptr(), _ptr(v), pages, heads, rows, d, *k.stride()[:3], *vs, _dtype_code(k))


def parallax_cache_fork(pages, parents, children, stream=None):
    """Sequence children[i] (empty) becomes a copy of parents[i] that shares its pages; see parallax_cache_fork in the header."""
    where = "parallax_cache_fork"
    device = _table_device(where, pages)
    n = parents.numel()
    ptrs = _int_list(where, "parents", parents, None, device), _int_list(where, "children", children, n, device)
    st = load_library().parallax_cache_fork(ctypes.byref(pages._args), *ptrs, n, _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)


def parallax_cache_extend(pages, seqs, new_lens, *pools, stream=None):
    """Room for new_lens[i] tokens in sequence seqs[i] (clamped to what it has and what its table row can hold): a page for every
    token that is new. pools: k, v (, k, v ...) of the layers that the table serves; shared last pages that are replaced are
    copied in all of them. Returns `missing` (int32 [1] on the device: 0, or how many pages were lacking, and then nothing was
    changed). Without pools (missing, src, dst, rows) is returned, and
    parallax_cache_copy(k, v, src, dst, rows) is the caller's to call for every layer."""
    where = "parallax_cache_extend"
    device = _table_device(where, pages)
    n = seqs.numel()
    ptrs = _int_list(where, "seqs", seqs, None, device), _int_list(where, "new_lens", new_lens, n, device)
    if len(pools) % 2:
        raise ValueError("pools come as k, v (v None: a single pool)")
    lib, where_to = load_library(), _launch_stream(where, stream)
    # Every layer's pools are looked at before the table changes: a refusal behind that would leave shared pages replaced whose
    # rows have not been copied. (A copy of nothing is checked like any other, and launches nothing.)
    layers = []
    for k, v in zip(pools[::2], pools[1::2]):
        a = _filled(plx_cache_pools, *_pools(where, k, v))
        if a.num_pages != pages.page_refs.numel() or a.page_size != pages.page_size:
            raise ValueError("the pools have the pages of the table")
        st = lib.parallax_cache_copy(ctypes.byref(a), 0, 0, 0, 0, where_to)
        if st != PLX_OK:
            raise ParallaxError(st, "parallax_cache_copy")
        layers.append(a)
    buf = _result_maker(stream, torch.empty)(3 * n + 1, dtype=torch.int32, device=pages.block_table.device)
    at = buf.data_ptr()
    src, dst, rows, missing = at, at + 4 * n, at + 8 * n, at + 12 * n
    st = lib.parallax_cache_extend(ctypes.byref(pages._args), *ptrs, n, src, dst, rows, missing, where_to)
    if st != PLX_OK:
        raise ParallaxError(st, where)
    for a in layers:
        st = lib.parallax_cache_copy(ctypes.byref(a), src, dst, rows, n, where_to)
        if st != PLX_OK:
            raise ParallaxError(st, "parallax_cache_copy")
    return buf[3 * n:] if pools else (buf[3 * n:], buf[:n], buf[n:2 * n], buf[2 * n:3 * n])


def parallax_cache_free(pages, seqs, first=None, last=None, stream=None):
    """Sequence seqs[i] gives back the whole pages in its tokens first[i] .. last[i] - 1 (default: all of them; a last[i] at or
    behind its length takes the partial last page along and shortens the sequence to first[i])."""
    where = "parallax_cache_free"
    device = _table_device(where, pages)
    n = seqs.numel()
    ptrs = [_int_list(where, "seqs", seqs, None, device)]
    ptrs += [0 if t is None else _int_list(where, name, t, n, device) for name, t in (("first", first), ("last", last))]
    st = load_library().parallax_cache_free(ctypes.byref(pages._args), *ptrs, n, _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)


def parallax_cache_copy(k, v, src, dst, rows=None, stream=None):
    """Page src[i] -> page dst[i] of the pools k and v (None: k only), its first rows[i] rows (default: all)."""
    where = "parallax_cache_copy"
    a = _filled(plx_cache_pools, *_pools(where, k, v))
    n = src.numel()
    ptrs = [_int_list(where, "src", src, None, _here()), _int_list(where, "dst", dst, n, _here())]
    ptrs.append(0 if rows is None else _int_list(where, "rows", rows, n, _here()))
    st = load_library().parallax_cache_copy(ctypes.byref(a), *ptrs, n, _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)


def parallax_cache_compact(k, v, seq_lens, draft_lens, accepted, n_accepted, block_table=None, new_lens=None, max_draft=None,
                           stream=None):
    """The rows of the accepted nodes (numbers accepted[b][: n_accepted[b]], ascending) among the last min(draft_lens[b], max_draft)
    cached ones (draft_lens None: max_draft) move together behind the committed rows. max_draft is the Tq of the tree that was verified (not
    given: 256, the same where no draft_lens[b] is above Tq). k, v: pools with a block_table, else [B, Hkv, capacity, d];
    v None: k only. Returns new_lens [B] = committed + accepted; seq_lens stays as it is."""
    where = "parallax_cache_compact"
    pools = _pools(where, k, v)
    if accepted.dim() != 2:
        raise ValueError("accepted [B, most]")
    B, most = accepted.shape
    if max_draft is None:
        if draft_lens is None:
            raise ValueError("draft_lens or max_draft is needed")
        max_draft = 256
    if new_lens is None:
        new_lens = _result_maker(stream, torch.empty)(B, dtype=torch.int32, device=k.device)
    here = k.get_device()
    ptrs = [0 if t is None else _int_list(where, name, t, m, here) for name, t, m in (
        ("seq_lens", seq_lens, B), ("draft_lens", draft_lens, B), ("accepted", accepted, B * most),
        ("n_accepted", n_accepted, B), ("new_lens", new_lens, B))]
    table, stride = 0, 0
    if block_table is not None:
        if block_table.dtype != torch.int32 or block_table.get_device() != here or block_table.stride(1) != 1:
            raise TypeError("block_table must be an int32 device tensor [B, pages per sequence]")
        if block_table.shape[0] != B:
            raise ValueError("block_table needs one row per sequence")
        table, stride = block_table.data_ptr(), block_table.stride(0) if B > 1 else block_table.shape[1]
    a = _filled(plx_cache_compact_args, *pools, table, *ptrs, B, stride, _i32(max_draft), most)
    st = load_library().parallax_cache_compact(ctypes.byref(a), _launch_stream(where, stream))
    if st != PLX_OK:
        raise ParallaxError(st, where)
    return new_lens


def parallax_util_copy(dst, src, stream=None):
    nbytes = src.numel() * src.element_size()
    st = load_library().parallax_util_copy(dst.data_ptr(), src.data_ptr(), nbytes,
                                           _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_util_copy")
    return dst


def parallax_util_read(src, sink, stream=None):
    nbytes = src.numel() * src.element_size()
    st = load_library().parallax_util_read(src.data_ptr(), nbytes, sink.data_ptr(),
                                           _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_util_read")
    return sink


def parallax_util_read_grid(src, sink, workgroups, nbytes=None, stream=None):
    """Plain read of the first nbytes of src (default: all of it) by `workgroups` workgroups."""
    if nbytes is None:
        nbytes = src.numel() * src.element_size()
    st = load_library().parallax_util_read_grid(src.data_ptr(), int(nbytes), sink.data_ptr(), int(workgroups),
                                                _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_util_read_grid")
    return sink


def parallax_util_mfma(workgroups, iters, sink, stream=None) -> float:
    """Register-only bf16 MFMA loop; returns the flops it performs. sink: >= workgroups * 1024 bytes."""
    if sink.numel() * sink.element_size() < workgroups * 1024:
        raise ValueError("sink too small")
    st = load_library().parallax_util_mfma(int(workgroups), int(iters), sink.data_ptr(), _stream_ptr(stream))
    if st != PLX_OK:
        raise ParallaxError(st, "parallax_util_mfma")
    return float(workgroups) * 4 * iters * 8 * 32768


def parallax_util_read_sink_slots() -> int:
    return int(load_library().parallax_util_read_sink_slots())
