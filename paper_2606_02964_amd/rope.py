"""Binding of ``include/msa_rope.h``: rotary positions, applied as the fresh keys
and values are written into the paged cache.

The functions carry the C names and are re-exported by the package.  Tensors are
checked as in ``tree.py``; those of rows ([rows, heads, d]) also for their sizes, and that
a head's channels lie together.
"""
from __future__ import annotations

import ctypes
import math

import numpy as np

from . import MSA_ERR_INVALID_ARG, MsaError, Plan, _addr, _bind, _check, _f32, _f64, _i32, _i64, _lib, _P, msa_plan_info
from .tree import BF16, INT32, Tensor, address, here, refuse_large, refuse_tensor, values_address

try:
    import torch
    FLOAT64, UINT8 = (torch.float64,), (torch.uint8,)
    E4M3 = (torch.uint8, torch.float8_e4m3fn, torch.int8)  # or its bits
except ImportError:
    FLOAT64 = UINT8 = E4M3 = ()

__all__ = ["MSA_ROPE_HALF", "MSA_ROPE_INTERLEAVED", "MSA_ROPE_SCALE_NONE", "MSA_ROPE_SCALE_LINEAR", "MSA_ROPE_SCALE_BASE",
           "MSA_ROPE_SCALE_TURNS", "MSA_ROPE_SCALE_PAIRS", "msa_rope", "msa_rope_scaling", "make_rope", "msa_rope_freqs",
           "msa_rope_append"]

MSA_ROPE_HALF, MSA_ROPE_INTERLEAVED = 0, 1
(MSA_ROPE_SCALE_NONE, MSA_ROPE_SCALE_LINEAR, MSA_ROPE_SCALE_BASE, MSA_ROPE_SCALE_TURNS,
 MSA_ROPE_SCALE_PAIRS) = range(5)

EXPORTED_ROPE = ("msa_rope_freqs", "msa_rope_append")


class msa_rope(ctypes.Structure):
    _fields_ = [("inv_freq", _P), ("rotary_dim", _i32), ("pairs", _i32), ("amplitude", _f32), ("reserved", _i32)]


class msa_rope_scaling(ctypes.Structure):
    _fields_ = [("base", _f64), ("kind", _i32), ("reserved", _i32), ("factor", _f64), ("original_len", _f64),
                ("low", _f64), ("high", _f64)]


_bind("msa_rope_freqs", [ctypes.POINTER(msa_rope_scaling), _i32, _P, ctypes.POINTER(_f32)])
_bind("msa_rope_append", [_P, _P, _P, _i64, _i64, _P, _i64, _i64, _P, _P, _i64, _i64, _i64, _i64, _P, _P, _P, _P, _P, _P,
                          _P])


def make_rope(inv_freq, pairs: int = MSA_ROPE_HALF, amplitude: float = 1.0) -> msa_rope:
    """How a model's channels are rotated: ``inv_freq`` is a float64 device tensor [rotary_dim / 2], which the
    returned object keeps."""
    if not hasattr(inv_freq, "data_ptr") or inv_freq.dtype not in FLOAT64 or inv_freq.dim() != 1 \
            or not inv_freq.is_contiguous() or not inv_freq.is_cuda:
        raise MsaError(MSA_ERR_INVALID_ARG, "make_rope: inv_freq is not a contiguous float64 vector on a GPU")
    rope = msa_rope(inv_freq.data_ptr(), 2 * inv_freq.shape[0], int(pairs), float(amplitude), 0)
    rope.tensor, rope.device = inv_freq, inv_freq.get_device()
    rope.address = ctypes.addressof(rope)
    return rope


def msa_rope_freqs(rotary_dim: int, base: float = 10000.0, kind: int = MSA_ROPE_SCALE_NONE, factor: float = 1.0,
                   original_len: float = 0.0, low: float = 1.0, high: float = 32.0):
    """(frequencies float64 [rotary_dim / 2], amplitude) on the host."""
    refuse_large("msa_rope_freqs", rotary_dim=int(rotary_dim), kind=int(kind))
    out, amplitude = np.zeros(max(1, int(rotary_dim) // 2)), _f32()
    scaling = msa_rope_scaling(base, int(kind), 0, factor, original_len, low, high)
    _check(_lib.msa_rope_freqs(ctypes.byref(scaling), int(rotary_dim), out.ctypes.data, ctypes.byref(amplitude)))
    return out, amplitude.value


def sizes(plan: Plan):
    """(rows, query heads, KV heads, d, entries of the block table, entries of a cache's powers of two)."""
    try:
        return plan.row_sizes
    except AttributeError:
        sh = plan.shape
        if not plan.handle or sh is None:  # no plan: the library reports that
            return 0, 0, 0, 0, 0, 0
        plan.row_sizes = (msa_plan_info(plan)["total_q"], sh.num_q_heads, sh.num_kv_heads, sh.head_dim,
                          sh.num_seqs * sh.max_blocks_per_seq, sh.num_blocks * sh.num_kv_heads * sh.block_size)
        return plan.row_sizes


def rows_of(who: str, name: str, x, rows: int, heads: int, d: int, dev: int):
    """(address, strides by row and head) of bfloat16 rows [rows, heads, d]; an address means contiguous ones."""
    if type(x) is Tensor and x.dtype in BF16 and x.get_device() == dev and x.dim() == 3:  # (a few reads, as in tree.py)
        n, h, c = x.shape
        if c == d and h == heads and n >= rows:
            if x.is_contiguous():
                return x.data_ptr(), h * d, d
            by_row, by_head, by_channel = x.stride()
            if by_channel == 1:  # (what a dimension of one entry says of its stride does not matter)
                return x.data_ptr(), by_row if n > 1 else h * d, by_head if h > 1 else d
    if x is None or type(x) is int or not hasattr(x, "stride"):
        return _addr(x), heads * d, d
    if x.dtype not in BF16 or x.get_device() != dev or not x.is_cuda:
        refuse_tensor(who, name, x, BF16, None, dev)
    if x.dim() != 3 or x.shape[0] < rows or x.shape[1] != heads or x.shape[2] != d:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} has shape {tuple(x.shape)}, ({rows}, {heads}, {d}) is needed")
    by_row, by_head, by_channel = x.stride()
    if by_channel != 1:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} is not contiguous along its last dimension")
    return x.data_ptr(), by_row if x.shape[0] > 1 else heads * d, by_head if heads > 1 else d


def bytes_address(who: str, name: str, x, dev: int):
    """Address of an 8-bit cache, which a shape's strides lay out; type and device are checked."""
    if type(x) is Tensor and x.dtype in E4M3 and x.get_device() == dev:
        return x.data_ptr()
    refuse_tensor(who, name, x, E4M3, None, dev)
    return _addr(x)


def msa_rope_append(plan: Plan, rope: msa_rope, q, q_out, k_new, v_new, block_table, k_cache, v_cache, k_scale=None,
                    v_scale=None, positions=None, stream=None) -> None:
    """Enqueue the rotation of ``q`` (bfloat16 [total_q, query heads, d], or None) into ``q_out`` and of ``k_new``
    ([total_q, KV heads, d]), and the write of K and ``v_new`` into the paged cache: a bfloat16 one, or with
    ``k_scale`` and ``v_scale`` (uint8 [blocks, KV heads, 16]) an 8-bit one.  ``positions`` int32 [total_q]: what the rows
    turn by (None: their positions in the plan)."""
    who = "msa_rope_append"
    dev, stream = here(stream)
    rows, hq, hkv, d, entries, powers = sizes(plan)
    if type(rope) is not msa_rope:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: rope is not an msa_rope")
    try:
        on, at = rope.device, rope.address
    except AttributeError:  # (not of make_rope)
        on, at = dev, ctypes.addressof(rope)
    if on != dev:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: rope's frequencies are on device {on}, the current device "
                                            f"is {dev}")
    qa, qt, qh = rows_of(who, "q", q, rows, hq, d, dev)
    oa, ot, oh = rows_of(who, "q_out", q_out, rows, hq, d, dev)
    ka, kt, kh = rows_of(who, "k_new", k_new, rows, hkv, d, dev)
    va, vt, vh = rows_of(who, "v_new", v_new, rows, hkv, d, dev)
    if k_scale is None and v_scale is None:
        kc, vc = values_address(who, "k_cache", k_cache, dev), values_address(who, "v_cache", v_cache, dev)
        ks = vs = None
    else:
        kc, vc = bytes_address(who, "k_cache", k_cache, dev), bytes_address(who, "v_cache", v_cache, dev)
        ks = address(who, "k_scale", k_scale, UINT8, powers, dev)
        vs = address(who, "v_scale", v_scale, UINT8, powers, dev)
    _check(_lib.msa_rope_append(plan.handle, at, qa, qt, qh, oa, ot, oh, ka, va, kt, kh, vt, vh,
                                None if positions is None else address(who, "positions", positions, INT32, rows, dev),
                                address(who, "block_table", block_table, INT32, entries, dev), kc, vc, ks, vs, stream))
