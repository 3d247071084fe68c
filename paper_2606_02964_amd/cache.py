"""Binding of ``include/msa_cache.h``: the attention weight each cached key has
received, the positions a reduced cache keeps, and their compaction.

The functions carry the C names and are re-exported by the package.  Tensor
arguments are checked for type, device and size; integer addresses are passed as
they are.
"""
from __future__ import annotations

import ctypes

try:
    import torch
except ImportError:  # the package itself does without
    torch = None

from . import MSA_ERR_INVALID_ARG, MsaError, Plan, _addr, _bind, _check, _i32, _i64, _lib, _P, _stream, msa_shape
from .tree import check_tensor

__all__ = ["msa_kv_weights", "msa_kv_weights_workspace", "msa_kv_select", "msa_kv_compact"]

EXPORTED_CACHE = tuple(__all__)

_bind("msa_kv_weights", [_P, _P, _P, _P, _P, _P, _i64, _i64, _i32, _P, ctypes.c_size_t, _P])
_bind("msa_kv_weights_workspace", [_P, ctypes.POINTER(ctypes.c_size_t)])
_bind("msa_kv_select", [_i32, _i32, _P, _i64, _i64, _i32, _P, _P, _i32, _i32, _i32, _P, _i64, _i64, _P, _P])
_bind("msa_kv_compact", [ctypes.POINTER(msa_shape), _P, _P, _i64, _i64, _i32, _P, _P, _P, _P, _P])


def _refuse(who: str, what: str) -> None:
    raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {what}")


def _lists(who: str, name: str, x, dtype: str, shape) -> None:
    """A tensor [sequences, lists, entries] of at least ``shape``, its entries contiguous."""
    if str(x.dtype)[6:] != dtype or not x.is_cuda:
        _refuse(who, f"{name} is not a {dtype} tensor on a GPU")
    if x.dim() != 3 or any(a < b for a, b in zip(x.shape, shape)):
        _refuse(who, f"{name} has shape {tuple(x.shape)}, {tuple(shape)} is needed")
    if x.shape[2] > 1 and x.stride(2) != 1:
        _refuse(who, f"{name} is not contiguous along its last dimension")


def _here(who: str, x) -> None:
    """Calls without a plan know no device of their own: their tensors are on the current one."""
    if x.device.index != torch.cuda.current_device():
        _refuse(who, f"tensors are on device {x.device.index}, the current device is {torch.cuda.current_device()}")


def msa_kv_weights_workspace(plan: Plan) -> int:
    """Bytes of workspace that ``msa_kv_weights`` needs (may be 0)."""
    out = ctypes.c_size_t()
    _check(_lib.msa_kv_weights_workspace(plan.handle, ctypes.byref(out)))
    return out.value


def msa_kv_weights(plan: Plan, q, k_cache, block_table, lse, weights, workspace=None, accumulate: bool = True,
                   stream=None) -> None:
    """Enqueue the sum of the plan's softmax weights by key into ``weights`` float32 [sequences, KV heads, positions];
    ``accumulate`` adds to what is there."""
    who, sh = "msa_kv_weights", plan.shape
    need = getattr(plan, "_positions", None)
    if need is None:  # the most positions a sequence may have
        need = plan._positions = sh.max_blocks_per_seq * sh.block_size
    _lists(who, "weights", weights, "float32", (sh.num_seqs, sh.num_kv_heads, need))
    size = 0 if workspace is None else int(workspace.numel() * workspace.element_size())
    _check(_lib.msa_kv_weights(plan.handle, _addr(q), _addr(k_cache), _addr(block_table), _addr(lse), _addr(weights),
                               weights.stride(0), weights.stride(1), int(accumulate), _addr(workspace), size,
                               _stream(stream)))


def msa_kv_select(scores, seq_len, keep, index, count, first: int = 0, recent: int = 0, stream=None) -> None:
    """Enqueue the choice of the positions that stay: ``scores`` float32 [sequences, lists, positions], ``seq_len`` and
    ``keep`` int32 [sequences]; ``index`` int32 [sequences, lists, entries] and ``count`` int32 [sequences] are
    written."""
    who = "msa_kv_select"
    if getattr(scores, "dim", lambda: 0)() != 3:
        _refuse(who, "scores is not a tensor [sequences, lists, positions]")
    B, H, L = scores.shape
    _lists(who, "scores", scores, "float32", (B, H, 0))
    _lists(who, "index", index, "int32", (B, H, 0))
    for name, x in (("seq_len", seq_len), ("keep", keep), ("count", count)):
        check_tensor(who, name, x, ("int32",), B)
    _here(who, scores)
    _check(_lib.msa_kv_select(B, H, _addr(scores), scores.stride(0), scores.stride(1), L, _addr(seq_len), _addr(keep),
                              int(first), int(recent), index.shape[2], _addr(index), index.stride(0), index.stride(1),
                              _addr(count), _stream(stream)))


def msa_kv_compact(shape: msa_shape, base, index, count, block_table, k_cache, v_cache, stream=None) -> None:
    """Enqueue the moves of K and V at ``base[b] + index[b, (head,) i]`` to ``base[b] + i``, i < ``count[b]``.
    ``index`` int32 [sequences, entries], the same for all heads, or [sequences, KV heads, entries]; ``base`` (or None:
    0) and ``count`` int32 [sequences]."""
    who, B = "msa_kv_compact", shape.num_seqs
    if index.dim() == 2:
        index = index[:, None].expand(-1, shape.num_kv_heads, -1)
    _lists(who, "index", index, "int32", (B, shape.num_kv_heads, 0))
    for name, x in (("base", base), ("count", count)):
        check_tensor(who, name, x, ("int32",), B)
    _here(who, index)
    _check(_lib.msa_kv_compact(ctypes.byref(shape), _addr(base), _addr(index), index.stride(0), index.stride(1),
                               index.shape[2], _addr(count), _addr(block_table), _addr(k_cache), _addr(v_cache),
                               _stream(stream)))
