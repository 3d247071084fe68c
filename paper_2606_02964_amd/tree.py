"""Binding of ``include/msa_tree.h``: attention of trees of drafted tokens over
the paged cache, and the verification of the drafts.

The functions carry the C names and are re-exported by the package.  Tensor
arguments are checked for type, device and size (the library sees addresses
only); integer addresses are passed as they are.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

from . import (MSA_ERR_INVALID_ARG, MSA_PLAN_HOST_ONLY, MsaError, Plan, _addr, _bind, _check, _host_i32, _i32, _i64,
               _lib, _P, _stream, msa_plan_opts, msa_shape)

__all__ = ["MSA_TREE_MAX_SLOTS", "MSA_PROB_F32", "MSA_PROB_BF16", "MSA_PROB_F16", "msa_tree_info_t", "msa_plan_tree",
           "msa_plan_tree_info", "msa_tree_mask", "msa_tree_forward", "msa_tree_verify", "msa_tree_verify_workspace"]

MSA_TREE_MAX_SLOTS = 1024
MSA_PROB_F32, MSA_PROB_BF16, MSA_PROB_F16 = 0, 1, 2


class msa_tree_info_t(ctypes.Structure):
    _fields_ = [("num_trees", _i64), ("tree_rows", _i64), ("max_slots", _i64), ("mask_words", _i64)]


EXPORTED_TREE = ("msa_plan_tree", "msa_plan_tree_info", "msa_tree_mask", "msa_tree_forward", "msa_tree_verify",
                 "msa_tree_verify_workspace")

_bind("msa_plan_tree", [ctypes.POINTER(msa_shape), _P, _P, _P, _P, _P, ctypes.POINTER(msa_plan_opts), _P,
                        ctypes.POINTER(_P)])
_bind("msa_plan_tree_info", [_P, ctypes.POINTER(msa_tree_info_t)])
_bind("msa_tree_mask", [_P, _P, _P, _i64, _P])
_bind("msa_tree_forward", [_P, _P, _P, _P, _P, _P, _i64, _P, _P, _P, ctypes.c_size_t, _P])
_bind("msa_tree_verify", [_P, _i32, _i32, _P, _i64, _P, _i64, _P, _P, _P, _P, _P, _i64, _P, _P, _P, ctypes.c_size_t,
                          _P])
_bind("msa_tree_verify_workspace", [_P, _i32, ctypes.POINTER(ctypes.c_size_t)])


def check_tensor(who: str, name: str, x, dtypes: Sequence[str], need: int, rows: Optional[int] = None) -> None:
    """Refuses a tensor of another type, on the host, not contiguous, or with fewer than ``need`` elements; with
    ``rows``, a 2-D one (rows, need) whose last dimension is contiguous.  Other objects pass."""
    if x is None or isinstance(x, int) or not hasattr(x, "stride"):
        return
    bad = None
    if str(x.dtype)[6:] not in dtypes:
        bad = f"has type {x.dtype}, not {' or '.join(dtypes)}"
    elif not x.is_cuda:
        bad = "is not on a GPU"
    elif rows is None:
        if not x.is_contiguous():
            bad = "is not contiguous"
        elif x.numel() < need:
            bad = f"has {x.numel()} elements, {need} are needed"
    elif x.dim() != 2 or x.shape[0] < rows or x.shape[1] < need:
        bad = f"has shape {tuple(x.shape)}, ({rows}, {need}) is needed"
    elif rows and x.stride(1) != 1 and need > 1:
        bad = "is not contiguous along its last dimension"
    if bad:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} {bad}")


def workspace_bytes(workspace, given: int) -> int:
    if workspace is None or given:
        return int(given)
    return int(workspace.numel() * workspace.element_size())


def _row_stride(x, given: Optional[int], width: int) -> int:
    if given is not None:
        return int(given)
    if hasattr(x, "stride") and x.dim() == 2:
        return int(x.stride(0)) if x.shape[0] > 1 else max(int(x.shape[1]), width)
    return width


def msa_plan_tree(shape: msa_shape, seq_kv_len: Sequence[int], seg_indptr: Sequence[int], seg_start: Sequence[int],
                  seg_len: Sequence[int], seg_tree: Optional[Sequence[int]] = None, q_tile_tokens: int = 0,
                  kv_split_tokens: int = 0, flags: int = 0, stream=None) -> Plan:
    """A plan some of whose segments are trees (``seg_tree`` 1; None: all of them)."""
    kv, ip, ss, sl = _host_i32(seq_kv_len), _host_i32(seg_indptr), _host_i32(seg_start), _host_i32(seg_len)
    tr = None if seg_tree is None else _host_i32(seg_tree)
    if tr is not None and tr.size != sl.size:
        raise MsaError(MSA_ERR_INVALID_ARG, f"msa_plan_tree: seg_tree has {tr.size} entries for {sl.size} segments")
    opts = msa_plan_opts(q_tile_tokens, kv_split_tokens, flags)
    handle = _P()
    _check(_lib.msa_plan_tree(ctypes.byref(shape), kv.ctypes.data, ip.ctypes.data,
                              ss.ctypes.data if ss.size else None, sl.ctypes.data if sl.size else None,
                              tr.ctypes.data if tr is not None and tr.size else None, ctypes.byref(opts),
                              None if flags & MSA_PLAN_HOST_ONLY else _stream(stream), ctypes.byref(handle)))
    plan = Plan(handle.value, shape)
    info = msa_plan_tree_info(plan)
    plan.trees, plan.tree_rows = info["num_trees"], info["tree_rows"]
    plan.max_slots, plan.mask_words = info["max_slots"], info["mask_words"]
    return plan


def msa_plan_tree_info(plan: Plan) -> dict:
    info = msa_tree_info_t()
    _check(_lib.msa_plan_tree_info(plan.handle, ctypes.byref(info)))
    return {name: getattr(info, name) for name, _ in info._fields_}


def _figures(plan: Plan):
    """(trees, tree rows, slots of the largest, mask words); zeros for a plan without trees, whose calls the library
    refuses or answers without reading anything."""
    return (getattr(plan, "trees", 0), getattr(plan, "tree_rows", 0), getattr(plan, "max_slots", 0),
            getattr(plan, "mask_words", 0))


def msa_tree_mask(plan: Plan, parents, mask, mask_stride: Optional[int] = None, stream=None) -> None:
    """Enqueue the trees' ancestor masks: ``parents`` int32 [tree_rows] to ``mask`` int64 or uint64
    [tree_rows, >= mask_words]."""
    _, rows, _, words = _figures(plan)
    check_tensor("msa_tree_mask", "parents", parents, ("int32",), rows)
    check_tensor("msa_tree_mask", "mask", mask, ("int64", "uint64"), words, rows)
    _check(_lib.msa_tree_mask(plan.handle, _addr(parents), _addr(mask), _row_stride(mask, mask_stride, words),
                              _stream(stream)))


def msa_tree_forward(plan: Plan, q, k_cache, v_cache, block_table, mask, o, lse=None, workspace=None,
                     workspace_bytes: int = 0, mask_stride: Optional[int] = None, stream=None) -> None:
    """Enqueue the attention of a plan with trees for one layer; ``mask`` as of ``msa_tree_mask`` (None if the plan
    has no tree), the rest as of ``msa_forward``."""
    _, rows, _, words = _figures(plan)
    check_tensor("msa_tree_forward", "mask", mask, ("int64", "uint64"), words, rows)
    if workspace is not None and not workspace_bytes:
        workspace_bytes = int(workspace.numel() * workspace.element_size())
    _check(_lib.msa_tree_forward(plan.handle, _addr(q), _addr(k_cache), _addr(v_cache), _addr(block_table),
                                 _addr(mask), _row_stride(mask, mask_stride, words), _addr(o), _addr(lse),
                                 _addr(workspace), int(workspace_bytes), _stream(stream)))


def msa_tree_verify_workspace(plan: Plan, vocab: int) -> int:
    """Bytes of workspace that ``msa_tree_verify`` needs."""
    out = ctypes.c_size_t()
    _check(_lib.msa_tree_verify_workspace(plan.handle, int(vocab), ctypes.byref(out)))
    return out.value


_PROB = {"float32": MSA_PROB_F32, "bfloat16": MSA_PROB_BF16, "float16": MSA_PROB_F16}


def msa_tree_verify(plan: Plan, target, tokens, parents, u_accept, u_sample, path, path_len, next_token, draft=None,
                    workspace=None, stream=None) -> None:
    """Enqueue the verification of the plan's trees.  ``target`` (and ``draft``, or None) are tensors
    [tree_rows, vocab] of float32, bfloat16 or float16; ``path`` int32 [trees, >= max_slots], ``path_len`` and
    ``next_token`` int32 [trees] are written."""
    who = "msa_tree_verify"
    trees, rows, slots, _ = _figures(plan)
    if target is None or target.dim() != 2:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: target is not a 2-D tensor")
    vocab, kind = int(target.shape[1]), str(target.dtype)[6:]
    check_tensor(who, "target", target, tuple(_PROB), vocab, rows)
    check_tensor(who, "draft", draft, (kind,), vocab, rows)
    for name, x, dtype, need in (("tokens", tokens, "int32", rows), ("parents", parents, "int32", rows),
                                 ("u_accept", u_accept, "float32", rows), ("u_sample", u_sample, "float32", trees),
                                 ("path_len", path_len, "int32", trees), ("next_token", next_token, "int32", trees)):
        check_tensor(who, name, x, (dtype,), need)
    check_tensor(who, "path", path, ("int32",), slots, trees)
    _check(_lib.msa_tree_verify(plan.handle, _PROB[kind], vocab, _addr(target), _row_stride(target, None, vocab),
                                _addr(draft), 0 if draft is None else _row_stride(draft, None, vocab), _addr(tokens),
                                _addr(parents), _addr(u_accept), _addr(u_sample), _addr(path),
                                _row_stride(path, None, slots), _addr(path_len), _addr(next_token), _addr(workspace),
                                workspace_bytes(workspace, 0), _stream(stream)))
