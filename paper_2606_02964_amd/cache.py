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
    # torch's own lookup takes 0.15 us, the public call 0.26
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
except ImportError:  # the package itself does without
    torch = None

from . import MSA_ERR_INVALID_ARG, MsaError, Plan, _addr, _bind, _check, _i32, _i64, _lib, _P, _stream, msa_shape
from .tree import FLOAT32, INT32, address, rows_address, size_of

__all__ = ["msa_kv_weights", "msa_kv_weights_workspace", "msa_kv_select", "msa_kv_compact"]

EXPORTED_CACHE = tuple(__all__)

_bind("msa_kv_weights", [_P, _P, _P, _P, _P, _P, _i64, _i64, _i32, _P, ctypes.c_size_t, _P])
_bind("msa_kv_weights_workspace", [_P, ctypes.POINTER(ctypes.c_size_t)])
_bind("msa_kv_select", [_i32, _i32, _P, _i64, _i64, _i32, _P, _P, _i32, _i32, _i32, _P, _i64, _i64, _P, _P])
_bind("msa_kv_compact", [ctypes.POINTER(msa_shape), _P, _P, _i64, _i64, _i32, _P, _P, _P, _P, _P])


def _refuse(who: str, what: str) -> None:
    raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {what}")


def _lists(who: str, name: str, x, dtypes, a: int, b: int, c: int):
    """(address, strides) of a tensor [sequences, lists, entries] of at least (a, b, c), its entries contiguous."""
    have, step = x.shape, x.stride()
    if x.dtype in dtypes and x.is_cuda and len(have) == 3 and have[0] >= a and have[1] >= b and have[2] >= c \
            and (step[2] == 1 or have[2] <= 1):
        return x.data_ptr(), step
    if x.dtype not in dtypes or not x.is_cuda:
        _refuse(who, f"{name} is not a {dtypes[0]} tensor on a GPU")
    if len(have) != 3 or have[0] < a or have[1] < b or have[2] < c:
        _refuse(who, f"{name} has shape {tuple(have)}, {(a, b, c)} is needed")
    _refuse(who, f"{name} is not contiguous along its last dimension")


def _here(who: str, x) -> None:
    """Calls without a plan know no device of their own: their tensors are on the current one."""
    if x.get_device() != _device():
        _refuse(who, f"tensors are on device {x.get_device()}, the current device is {_device()}")


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
    need = getattr(plan, "positions", None)
    if need is None:  # the most positions a sequence may have
        need = plan.positions = sh.max_blocks_per_seq * sh.block_size
        plan.heads = (sh.num_seqs, sh.num_kv_heads)
    at, step = _lists(who, "weights", weights, FLOAT32, *plan.heads, need)
    _check(_lib.msa_kv_weights(plan.handle, _addr(q), _addr(k_cache), _addr(block_table), _addr(lse), at, step[0],
                               step[1], int(accumulate), _addr(workspace), size_of(workspace), _stream(stream)))


def msa_kv_select(scores, seq_len, keep, index, count, first: int = 0, recent: int = 0, stream=None) -> None:
    """Enqueue the choice of the positions that stay: ``scores`` float32 [sequences, lists, positions], ``seq_len`` and
    ``keep`` int32 [sequences]; ``index`` int32 [sequences, lists, entries] and ``count`` int32 [sequences] are
    written."""
    who = "msa_kv_select"
    if len(getattr(scores, "shape", ())) != 3:
        _refuse(who, "scores is not a tensor [sequences, lists, positions]")
    B, H, L = scores.shape
    at, step = _lists(who, "scores", scores, FLOAT32, B, H, 0)
    to, to_step = _lists(who, "index", index, INT32, B, H, 0)
    _here(who, scores)
    _check(_lib.msa_kv_select(B, H, at, step[0], step[1], L, address(who, "seq_len", seq_len, INT32, B),
                              address(who, "keep", keep, INT32, B), int(first), int(recent), index.shape[2], to,
                              to_step[0], to_step[1], address(who, "count", count, INT32, B), _stream(stream)))


def msa_kv_compact(shape: msa_shape, base, index, count, block_table, k_cache, v_cache, stream=None) -> None:
    """Enqueue the moves of K and V at ``base[b] + index[b, (head,) i]`` to ``base[b] + i``, i < ``count[b]``.
    ``index`` int32 [sequences, entries], the same for all heads, or [sequences, KV heads, entries]; ``base`` (or None:
    0) and ``count`` int32 [sequences]."""
    who, B = "msa_kv_compact", shape.num_seqs
    if index.dim() == 2:
        entries = index.shape[1]
        at, _ = rows_address(who, "index", index, INT32, entries, B)
        per_seq, per_head = index.stride(0), 0
    else:
        at, (per_seq, per_head, _) = _lists(who, "index", index, INT32, B, shape.num_kv_heads, 0)
        entries = index.shape[2]
    _here(who, index)
    _check(_lib.msa_kv_compact(ctypes.byref(shape), address(who, "base", base, INT32, B), at, per_seq, per_head, entries,
                               address(who, "count", count, INT32, B), _addr(block_table), _addr(k_cache),
                               _addr(v_cache), _stream(stream)))
