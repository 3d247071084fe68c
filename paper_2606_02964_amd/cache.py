"""Binding of ``include/msa_cache.h``: the attention weight each cached key has
received, the positions a reduced cache keeps, and their compaction.

The functions carry the C names and are re-exported by the package.  Tensors
are checked as in ``tree.py``: type, device, and size and layout, except where a
shape's strides give those (q and the caches).  Integer addresses are passed as
they are, where a function does not ask for a tensor.
"""
from __future__ import annotations

import ctypes

from . import MSA_ERR_INVALID_ARG, MsaError, Plan, _bind, _check, _i32, _i64, _lib, _P, msa_shape
from .tree import (FLOAT32, INT32, address, here, refuse_large, refuse_tensor, rows_address, sizes_of, values_address,
                   workspace_of)

__all__ = ["msa_kv_weights", "msa_kv_weights_workspace", "msa_kv_select", "msa_kv_compact"]

EXPORTED_CACHE = tuple(__all__)

_bind("msa_kv_weights", [_P, _P, _P, _P, _P, _P, _i64, _i64, _i32, _P, ctypes.c_size_t, _P])
_bind("msa_kv_weights_workspace", [_P, ctypes.POINTER(ctypes.c_size_t)])
_bind("msa_kv_select", [_i32, _i32, _P, _i64, _i64, _i32, _P, _P, _i32, _i32, _i32, _P, _i64, _i64, _P, _P])
_bind("msa_kv_compact", [ctypes.POINTER(msa_shape), _P, _P, _i64, _i64, _i32, _P, _P, _P, _P, _P])


def _refuse(who: str, what: str) -> None:
    raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {what}")


def _lists(who: str, name: str, x, dtypes, a: int, b: int, c: int, dev: int):
    """(address, strides) of a tensor [sequences, lists, entries] of at least (a, b, c), its entries contiguous."""
    try:
        have, step = x.shape, x.stride()
        if x.dtype in dtypes and x.get_device() == dev and have[0] >= a and have[1] >= b and have[2] >= c \
                and (step[2] == 1 or have[2] <= 1) and len(have) == 3:
            return x.data_ptr(), step
    except (AttributeError, IndexError):
        _refuse(who, f"{name} is not a tensor [sequences, lists, entries]")
    if len(have) != 3:
        _refuse(who, f"{name} is not a tensor [sequences, lists, entries]")
    refuse_tensor(who, name, x, dtypes, None, dev)
    if have[0] < a or have[1] < b or have[2] < c:
        _refuse(who, f"{name} has shape {tuple(have)}, {(a, b, c)} is needed")
    _refuse(who, f"{name} is not contiguous along its last dimension")


def msa_kv_weights_workspace(plan: Plan) -> int:
    """Bytes of workspace that ``msa_kv_weights`` needs (may be 0)."""
    out = ctypes.c_size_t()
    _check(_lib.msa_kv_weights_workspace(plan.handle, ctypes.byref(out)))
    return out.value


def msa_kv_weights(plan: Plan, q, k_cache, block_table, lse, weights, workspace=None, accumulate: bool = True,
                   stream=None, workspace_bytes: int = 0) -> None:
    """Enqueue the sum of the plan's softmax weights by key into the tensor ``weights`` float32 [sequences, KV heads,
    positions]; ``accumulate`` adds to what is there.  ``lse`` float32 [total_q, query heads] is that of msa_forward."""
    who = "msa_kv_weights"
    dev, stream = here(stream)
    entries, lses, seqs, heads, positions = sizes_of(plan)
    at, step = _lists(who, "weights", weights, FLOAT32, seqs, heads, positions, dev)
    ws, ws_bytes = workspace_of(who, workspace, workspace_bytes, dev)
    _check(_lib.msa_kv_weights(plan.handle, values_address(who, "q", q, dev),
                               values_address(who, "k_cache", k_cache, dev),
                               address(who, "block_table", block_table, INT32, entries, dev),
                               address(who, "lse", lse, FLOAT32, lses, dev), at, step[0], step[1], int(accumulate),
                               ws, ws_bytes, stream))


def msa_kv_select(scores, seq_len, keep, index, count, first: int = 0, recent: int = 0, stream=None) -> None:
    """Enqueue the choice of the positions that stay: tensors ``scores`` float32 [sequences, lists, positions] and
    ``index`` int32 [sequences, lists, entries]; ``seq_len`` and ``keep`` int32 [sequences].  ``index`` and ``count``
    int32 [sequences] are written."""
    who = "msa_kv_select"
    dev, stream = here(stream)
    if len(getattr(scores, "shape", ())) != 3:
        _refuse(who, "scores is not a tensor [sequences, lists, positions]")
    B, H, L = scores.shape
    at, step = _lists(who, "scores", scores, FLOAT32, B, H, 0, dev)
    to, to_step = _lists(who, "index", index, INT32, B, H, 0, dev)
    first, recent, entries = int(first), int(recent), index.shape[2]
    if (first | recent | B | H | L | entries) >> 31:  # (negative ones too)
        refuse_large(who, first=first, recent=recent, sequences=B, lists=H, positions=L, entries=entries)
    _check(_lib.msa_kv_select(B, H, at, step[0], step[1], L, address(who, "seq_len", seq_len, INT32, B, dev),
                              address(who, "keep", keep, INT32, B, dev), first, recent, entries, to,
                              to_step[0], to_step[1], address(who, "count", count, INT32, B, dev), stream))


def msa_kv_compact(shape: msa_shape, base, index, count, block_table, k_cache, v_cache, stream=None) -> None:
    """Enqueue the moves of K and V at ``base[b] + index[b, (head,) i]`` to ``base[b] + i``, i < ``count[b]``.
    ``index`` is an int32 tensor [sequences, entries], the same for all heads, or [sequences, KV heads, entries];
    ``base`` (or None: 0) and ``count`` int32 [sequences], ``block_table`` int32 [sequences, max_blocks_per_seq]."""
    who, B = "msa_kv_compact", shape.num_seqs
    dev, stream = here(stream)
    if not hasattr(index, "stride"):
        _refuse(who, "index is not a tensor")
    if index.dim() == 2:
        entries = index.shape[1]
        at, per_seq = rows_address(who, "index", index, INT32, entries, B, dev)
        per_head = 0
    else:
        at, (per_seq, per_head, _) = _lists(who, "index", index, INT32, B, shape.num_kv_heads, 0, dev)
        entries = index.shape[2]
    if entries >> 31:
        refuse_large(who, entries=entries)
    _check(_lib.msa_kv_compact(ctypes.byref(shape), address(who, "base", base, INT32, B, dev), at, per_seq, per_head,
                               entries, address(who, "count", count, INT32, B, dev),
                               address(who, "block_table", block_table, INT32, B * shape.max_blocks_per_seq, dev),
                               values_address(who, "k_cache", k_cache, dev),
                               values_address(who, "v_cache", v_cache, dev), stream))
