"""Binding of ``include/msa_fp8.h``: the paged cache in 8 bits, written as it is
quantised, attended to, and read back into a bfloat16 cache.

The functions carry the C names and are re-exported by the package.  Tensors are
checked as in ``tree.py`` and ``rope.py``; the 8-bit caches are uint8 or float8_e4m3fn, their
powers of two uint8 [blocks, KV heads, 16].
"""
from __future__ import annotations

import ctypes
from typing import Optional

from . import Plan, _bind, _check, _i32, _i64, _lib, _P, msa_shape
from .rope import UINT8, bytes_address, rows_of, sizes
from .tree import FLOAT32, INT32, address, here, refuse_large, values_address, workspace_of

__all__ = ["msa_fp8_append", "msa_fp8_forward", "msa_fp8_read"]

EXPORTED_FP8 = tuple(__all__)

_bind("msa_fp8_append", [_P, _P, _P, _i64, _i64, _i64, _i64, _P, _P, _P, _P, _P, _P])
_bind("msa_fp8_forward", [_P, _P, _P, _P, _P, _P, _P, _P, _P, _P, ctypes.c_size_t, _P])
_bind("msa_fp8_read", [ctypes.POINTER(msa_shape), _P, _P, _i32, _P, _P, _P, _P, _P, ctypes.POINTER(msa_shape), _P, _P, _P,
                       _P])


def msa_fp8_append(plan: Plan, k_new, v_new, block_table, k_cache, v_cache, k_scale, v_scale, stream=None) -> None:
    """Enqueue the write of the rows' fresh K/V (bfloat16 [total_q, KV heads, d]) into the 8-bit cache."""
    who = "msa_fp8_append"
    dev, stream = here(stream)
    rows, _, heads, d, entries, powers = sizes(plan)
    ka, kt, kh = rows_of(who, "k_new", k_new, rows, heads, d, dev)
    va, vt, vh = rows_of(who, "v_new", v_new, rows, heads, d, dev)
    _check(_lib.msa_fp8_append(plan.handle, ka, va, kt, kh, vt, vh,
                               address(who, "block_table", block_table, INT32, entries, dev),
                               bytes_address(who, "k_cache", k_cache, dev), bytes_address(who, "v_cache", v_cache, dev),
                               address(who, "k_scale", k_scale, UINT8, powers, dev),
                               address(who, "v_scale", v_scale, UINT8, powers, dev), stream))


def msa_fp8_forward(plan: Plan, q, k_cache, v_cache, k_scale, v_scale, block_table, o, lse=None, workspace=None,
                    workspace_bytes: int = 0, stream=None) -> None:
    """Enqueue MSA for one layer over the 8-bit cache; the rest as of ``msa_forward``."""
    who = "msa_fp8_forward"
    dev, stream = here(stream)
    rows, heads, _, _, entries, powers = sizes(plan)
    ws, ws_bytes = workspace_of(who, workspace, workspace_bytes, dev)
    _check(_lib.msa_fp8_forward(plan.handle, values_address(who, "q", q, dev),
                                bytes_address(who, "k_cache", k_cache, dev),
                                bytes_address(who, "v_cache", v_cache, dev),
                                address(who, "k_scale", k_scale, UINT8, powers, dev),
                                address(who, "v_scale", v_scale, UINT8, powers, dev),
                                address(who, "block_table", block_table, INT32, entries, dev),
                                values_address(who, "o", o, dev),
                                None if lse is None else address(who, "lse", lse, FLOAT32, rows * heads, dev), ws, ws_bytes,
                                stream))


def msa_fp8_read(shape: msa_shape, start, end, max_len: int, block_table, k_cache, v_cache, k_scale, v_scale,
                 to: msa_shape, to_table, k_out, v_out, stream: Optional[int] = None) -> None:
    """Enqueue the copy of positions ``start[b]`` (or None: 0) .. ``end[b]`` - 1, below ``max_len``, of the 8-bit
    cache of ``shape`` into the bfloat16 cache of ``to``, through each one's block table (int32 [sequences,
    max_blocks_per_seq]); ``start`` and ``end`` int32 [sequences]."""
    who, B = "msa_fp8_read", shape.num_seqs
    dev, stream = here(stream)
    max_len = int(max_len)
    if max_len >> 31:
        refuse_large(who, max_len=max_len)
    powers = shape.num_blocks * shape.num_kv_heads * 16
    _check(_lib.msa_fp8_read(ctypes.byref(shape), None if start is None else address(who, "start", start, INT32, B, dev),
                             address(who, "end", end, INT32, B, dev), max_len,
                             address(who, "block_table", block_table, INT32, B * shape.max_blocks_per_seq, dev),
                             bytes_address(who, "k_cache", k_cache, dev), bytes_address(who, "v_cache", v_cache, dev),
                             address(who, "k_scale", k_scale, UINT8, powers, dev),
                             address(who, "v_scale", v_scale, UINT8, powers, dev), ctypes.byref(to),
                             address(who, "to_table", to_table, INT32, B * to.max_blocks_per_seq, dev),
                             values_address(who, "k_out", k_out, dev), values_address(who, "v_out", v_out, dev), stream))
