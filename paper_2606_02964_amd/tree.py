"""Binding of ``include/msa_tree.h``: attention of trees of drafted tokens over
the paged cache, and the verification of the drafts.

The functions carry the C names and are re-exported by the package.  The library
sees addresses only, so tensors are checked here, and refused with MsaError: their
type, that they are on the current device (the library compares it with the
plan's), and their size and layout, except where a shape's strides give those: of
q, o and the caches.  Integer addresses are passed as they are, where a function
does not ask for a tensor.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Sequence

try:
    import torch
    Tensor = torch.Tensor
    INT32, FLOAT32, MASK = (torch.int32,), (torch.float32,), (torch.int64, torch.uint64)
    BF16 = (torch.bfloat16, torch.int16, torch.uint16)  # or its bits
    # torch's own lookups take 0.15 us, the public calls 0.26 and 2.9
    _device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    _raw_stream, _ready = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.is_initialized
    _PROB = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}  # MSA_PROB_*
except ImportError:  # the package itself does without; then nothing here is a tensor
    Tensor = None
    INT32 = FLOAT32 = MASK = BF16 = ()
    _PROB = {}

from . import (MSA_ERR_INVALID_ARG, MSA_PLAN_HOST_ONLY, MsaError, Plan, _addr, _bind, _check, _host_i32, _i32, _i64,
               _lib, _P, _stream, msa_plan_info, msa_plan_opts, msa_shape)

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


def here(stream):
    """(current device, handle of ``stream`` or of the device's current one); device -2, which no tensor is on, where
    there is none."""
    try:
        dev = _device()
    except (NameError, RuntimeError):
        return -2, _stream(stream)
    return dev, _raw_stream(dev) if stream is None and _raw_stream and _ready() else _stream(stream)


def refuse_tensor(who: str, name: str, x, dtypes, need: Optional[int], dev: int, rows: Optional[int] = None) -> None:
    """Refuses a tensor of another type, not on device ``dev``, not contiguous, or with fewer than ``need`` elements
    (None: any number, with any strides); with ``rows``, a 2-D one (rows, need) whose last dimension is contiguous.
    Other objects pass."""
    if x is None or type(x) is int or not hasattr(x, "stride"):
        return
    if x.dtype not in dtypes:
        bad = f"has type {x.dtype}, not {' or '.join(str(d) for d in dtypes)}"
    elif not x.is_cuda:
        bad = "is not on a GPU"
    elif x.get_device() != dev:
        bad = f"is on device {x.get_device()}, the current device is {dev}"
    elif need is None:
        return
    elif rows is not None and (x.dim() != 2 or x.shape[0] < rows or x.shape[1] < need):
        bad = f"has shape {tuple(x.shape)}, ({rows}, {need}) is needed"
    elif rows is not None:
        if need <= 1 or rows == 0 or x.stride(1) == 1:
            return
        bad = "is not contiguous along its last dimension"
    elif x.numel() < need:
        bad = f"has {x.numel()} elements, {need} are needed"
    else:
        if x.is_contiguous():
            return
        bad = "is not contiguous"
    raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} {bad}")


def address(who: str, name: str, x, dtypes, need: int, dev: int) -> Optional[int]:
    """Address of a tensor, checked as in ``refuse_tensor``, or of another object.  (These checks run on every call,
    which may be as short as a launch: the common case is a few attribute reads.)"""
    if type(x) is Tensor and x.dtype in dtypes and x.get_device() == dev and x.numel() >= need and x.is_contiguous():
        return x.data_ptr()
    refuse_tensor(who, name, x, dtypes, need, dev)
    return _addr(x)


def values_address(who: str, name: str, x, dev: int) -> Optional[int]:
    """Address of bfloat16 values that a shape's strides lay out; type and device are checked."""
    if type(x) is Tensor and x.dtype in BF16 and x.get_device() == dev:
        return x.data_ptr()
    refuse_tensor(who, name, x, BF16, None, dev)
    return _addr(x)


def rows_address(who: str, name: str, x, dtypes, need: int, rows: int, dev: int, given: Optional[int] = None):
    """(address, elements from row to row) of a 2-D tensor, checked likewise; ``given``: the latter, where it is."""
    if type(x) is Tensor and x.dtype in dtypes and x.get_device() == dev and x.dim() == 2:
        have, step = x.shape, x.stride()
        if have[0] >= rows and have[1] >= need and (step[1] == 1 or need <= 1 or rows == 0) and given is None:
            return x.data_ptr(), (step[0] if have[0] > 1 else max(have[1], need))
    refuse_tensor(who, name, x, dtypes, need, dev, rows)
    step = _row_stride(x, need)
    if given is not None and rows > 1 and hasattr(x, "stride") and int(given) != step:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} has {step} elements from row to row, not {int(given)}")
    return _addr(x), step if given is None else int(given)


def workspace_of(who: str, workspace, given: int, dev: int):
    """(address, bytes) of a workspace: a tensor, whose bytes are taken from it unless given, or an address."""
    if workspace is None:
        return None, int(given)
    if type(workspace) is not Tensor and not hasattr(workspace, "stride"):
        if not given:
            raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: workspace_bytes is needed with a workspace's address")
        return _addr(workspace), int(given)
    have = workspace.numel() * workspace.element_size()
    if workspace.get_device() != dev or not workspace.is_contiguous() or have < given:
        refuse_tensor(who, "workspace", workspace, (workspace.dtype,), -(-int(given) // workspace.element_size()), dev)
    return workspace.data_ptr(), int(given) or have


def refuse_large(who: str, **sizes: int) -> None:
    """Refuses sizes that the library's 32-bit arguments do not hold (ctypes would cut them off)."""
    for name, x in sizes.items():
        if not -1 << 31 <= x < 1 << 31:
            raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: {name} {x} does not fit 32 bits")


def sizes_of(plan: Plan):
    """(entries of the plan's block table, of its lse, its sequences, its KV heads, the most positions of a sequence)."""
    try:
        return plan.sizes
    except AttributeError:
        sh = plan.shape
        if not plan.handle or sh is None:  # no plan: the library reports that
            return 0, 0, 0, 0, 0
        plan.sizes = (sh.num_seqs * sh.max_blocks_per_seq, msa_plan_info(plan)["total_q"] * sh.num_q_heads, sh.num_seqs,
                      sh.num_kv_heads, sh.max_blocks_per_seq * sh.block_size)
        return plan.sizes


def _row_stride(x, width: int) -> int:
    if hasattr(x, "stride") and x.dim() == 2:
        return x.stride(0) if x.shape[0] > 1 else max(x.shape[1], width)
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
    plan.tree_rows, plan.max_slots, plan.mask_words = info["tree_rows"], info["max_slots"], info["mask_words"]
    plan.tree_figures = (info["num_trees"], info["tree_rows"], info["max_slots"], info["mask_words"])
    return plan


def msa_plan_tree_info(plan: Plan) -> dict:
    info = msa_tree_info_t()
    _check(_lib.msa_plan_tree_info(plan.handle, ctypes.byref(info)))
    return {name: getattr(info, name) for name, _ in info._fields_}


def _figures(plan: Plan):
    """(trees, tree rows, slots of the largest, mask words); zeros for a plan without trees, whose calls the library
    refuses or answers without reading anything."""
    return getattr(plan, "tree_figures", (0, 0, 0, 0))


def msa_tree_mask(plan: Plan, parents, mask, mask_stride: Optional[int] = None, stream=None) -> None:
    """Enqueue the trees' ancestor masks: ``parents`` int32 [tree_rows] to ``mask`` int64 or uint64
    [tree_rows, >= mask_words]."""
    _, rows, _, words = _figures(plan)
    dev, stream = here(stream)
    up = address("msa_tree_mask", "parents", parents, INT32, rows, dev)
    at, step = rows_address("msa_tree_mask", "mask", mask, MASK, words, rows, dev, mask_stride)
    _check(_lib.msa_tree_mask(plan.handle, up, at, step, stream))


def msa_tree_forward(plan: Plan, q, k_cache, v_cache, block_table, mask, o, lse=None, workspace=None,
                     workspace_bytes: int = 0, mask_stride: Optional[int] = None, stream=None) -> None:
    """Enqueue the attention of a plan with trees for one layer; ``mask`` as of ``msa_tree_mask`` (None if the plan
    has no tree), ``block_table`` int32 [sequences, max_blocks_per_seq], ``lse`` float32 [total_q, query heads], the rest
    as of ``msa_forward``."""
    who = "msa_tree_forward"
    dev, stream = here(stream)
    entries, lses = sizes_of(plan)[:2]
    _, rows, _, words = _figures(plan)
    at, step = rows_address(who, "mask", mask, MASK, words, rows, dev, mask_stride)
    ws, ws_bytes = workspace_of(who, workspace, workspace_bytes, dev)
    _check(_lib.msa_tree_forward(plan.handle, values_address(who, "q", q, dev),
                                 values_address(who, "k_cache", k_cache, dev),
                                 values_address(who, "v_cache", v_cache, dev),
                                 address(who, "block_table", block_table, INT32, entries, dev), at, step,
                                 values_address(who, "o", o, dev),
                                 None if lse is None else address(who, "lse", lse, FLOAT32, lses, dev), ws, ws_bytes,
                                 stream))


def msa_tree_verify_workspace(plan: Plan, vocab: int) -> int:
    """Bytes of workspace that ``msa_tree_verify`` needs."""
    out = ctypes.c_size_t()
    refuse_large("msa_tree_verify_workspace", vocab=int(vocab))
    _check(_lib.msa_tree_verify_workspace(plan.handle, int(vocab), ctypes.byref(out)))
    return out.value


def msa_tree_verify(plan: Plan, target, tokens, parents, u_accept, u_sample, path, path_len, next_token, draft=None,
                    workspace=None, stream=None, workspace_bytes: int = 0) -> None:
    """Enqueue the verification of the plan's trees.  ``target`` (and ``draft``, or None) are tensors
    [tree_rows, vocab] of float32, bfloat16 or float16; ``path`` int32 [trees, >= max_slots], ``path_len`` and
    ``next_token`` int32 [trees] are written."""
    who = "msa_tree_verify"
    dev, stream = here(stream)
    trees, rows, slots, _ = _figures(plan)
    if not hasattr(target, "stride") or target.dim() != 2:
        raise MsaError(MSA_ERR_INVALID_ARG, f"{who}: target is not a 2-D tensor")
    vocab, kind = target.shape[1], target.dtype
    if vocab >> 31:
        refuse_large(who, vocab=vocab)
    p, p_step = rows_address(who, "target", target, _PROB, vocab, rows, dev)
    q, q_step = (None, 0) if draft is None else rows_address(who, "draft", draft, (kind,), vocab, rows, dev)
    at, step = rows_address(who, "path", path, INT32, slots, trees, dev)
    ws, ws_bytes = workspace_of(who, workspace, workspace_bytes, dev)
    _check(_lib.msa_tree_verify(plan.handle, _PROB[kind], vocab, p, p_step, q, q_step,
                                address(who, "tokens", tokens, INT32, rows, dev),
                                address(who, "parents", parents, INT32, rows, dev),
                                address(who, "u_accept", u_accept, FLOAT32, rows, dev),
                                address(who, "u_sample", u_sample, FLOAT32, trees, dev), at, step,
                                address(who, "path_len", path_len, INT32, trees, dev),
                                address(who, "next_token", next_token, INT32, trees, dev), ws, ws_bytes,
                                stream))
