"""Binding of ``include/msa_window.h``: plans whose rows see a sliding window and
sinks.  The function carries the C name and is re-exported by the package."""
from __future__ import annotations

import ctypes
from typing import Sequence

from . import (MSA_PLAN_HOST_ONLY, Plan, _bind, _check, _host_i32, _i32, _lib, _P, _stream, msa_plan_opts, msa_shape)
from .tree import refuse_large

__all__ = ["msa_plan_window"]

EXPORTED_WINDOW = tuple(__all__)

_bind("msa_plan_window", [ctypes.POINTER(msa_shape), _P, _P, _P, _P, _i32, _i32, ctypes.POINTER(msa_plan_opts), _P,
                          ctypes.POINTER(_P)])


def msa_plan_window(shape: msa_shape, seq_kv_len: Sequence[int], seg_indptr: Sequence[int], seg_start: Sequence[int],
                    seg_len: Sequence[int], window: int, sinks: int = 0, q_tile_tokens: int = 0,
                    kv_split_tokens: int = 0, flags: int = 0, stream=None) -> Plan:
    """A plan whose rows see the latest ``window`` positions up to their own and the first ``sinks``; it goes into
    ``msa_forward``, ``msa_fp8_forward``, ``msa_kv_append`` and the others as any plan does."""
    kv, ip, ss, sl = _host_i32(seq_kv_len), _host_i32(seg_indptr), _host_i32(seg_start), _host_i32(seg_len)
    window, sinks = int(window), int(sinks)
    refuse_large("msa_plan_window", window=window, sinks=sinks)
    opts = msa_plan_opts(q_tile_tokens, kv_split_tokens, flags)
    handle = _P()
    _check(_lib.msa_plan_window(ctypes.byref(shape), kv.ctypes.data, ip.ctypes.data,
                                ss.ctypes.data if ss.size else None, sl.ctypes.data if sl.size else None, window, sinks,
                                ctypes.byref(opts), None if flags & MSA_PLAN_HOST_ONLY else _stream(stream),
                                ctypes.byref(handle)))
    return Plan(handle.value, shape)
