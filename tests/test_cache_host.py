"""Host side of msa_cache.h and msa_tree_verify (no GPU): declarations and refusals.
Addresses given here are never read: every call is refused, or has nothing to do."""
import ctypes
import os
import re

import pytest

import paper_2606_02964_amd as msa
from paper_2606_02964_amd import cache as C

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INV, UNS, OK = msa.MSA_ERR_INVALID_ARG, msa.MSA_ERR_UNSUPPORTED, msa.MSA_OK
P = 4096  # an address
lib = msa._lib


def shape(num_seqs=2, **kw):
    a = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=200, num_blocks=400, scale=0.1)
    a.update(kw)
    return msa.make_shape(num_seqs, **a)


def expect(status, text, got):
    assert got == status and text in msa.msa_last_error(), (got, msa.msa_last_error())


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "msa_cache.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(msa_[a-z_]+)\s*\(", text))
    assert names == set(C.EXPORTED_CACHE)
    loaded = ctypes.CDLL(msa.LIB_PATH)
    for n in names:
        assert hasattr(loaded, n) and hasattr(msa, n)


def test_headers_are_plain_c(tmp_path):
    import subprocess
    src = tmp_path / "c.c"
    src.write_text('#include "msa_tree.h"\n#include "msa_cache.h"\nint main(void) { return MSA_OK; }\n')
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-fsyntax-only", "-I",
                           os.path.join(ROOT, "include"), str(src)])


def test_weights_refusals():
    plan = msa.msa_plan(shape(), [500, 300], [0, 1, 2], [10, 200], [20, 100], flags=msa.MSA_PLAN_HOST_ONLY)
    trees = msa.msa_plan_tree(shape(), [500, 300], [0, 1, 2], [10, 200], [20, 100], flags=msa.MSA_PLAN_HOST_ONLY)
    call = lambda h=plan.handle, ss=9000, sh=3200, acc=1: lib.msa_kv_weights(h, P, P, P, P, P, ss, sh, acc, None, 0, None)  # noqa: E731
    expect(INV, "null plan", call(None))
    expect(UNS, "msa_plan_tree", call(trees.handle))
    expect(INV, "strides", call(ss=-1))
    expect(INV, "strides", call(sh=-8))
    expect(INV, "accumulate", call(acc=2))
    expect(INV, "HOST_ONLY", call())
    expect(INV, "null", lib.msa_kv_weights_workspace(None, None))


def test_select_refusals():
    def call(b=2, h=3, scores=P, ss=100, sl=30, ml=30, n=P, keep=P, first=1, recent=1, mk=9, index=P, is_=27, il=9, count=P):
        return lib.msa_kv_select(b, h, scores, ss, sl, ml, n, keep, first, recent, mk, index, is_, il, count, None)
    for kw in (dict(b=-1), dict(h=-1), dict(ml=-1), dict(first=-1), dict(recent=-1), dict(mk=-1)):
        expect(INV, "sizes", call(**kw))
    for kw in (dict(ss=-1), dict(sl=-1), dict(is_=-1), dict(il=-1)):
        expect(INV, "strides", call(**kw))
    for kw in (dict(scores=None), dict(n=None), dict(keep=None), dict(index=None), dict(count=None)):
        expect(INV, "non-null", call(**kw))
    for kw in (dict(scores=P + 2), dict(n=P + 1), dict(keep=P + 3), dict(index=P + 2), dict(count=P + 2)):
        expect(INV, "aligned", call(**kw))
    expect(UNS, "too many", call(b=1 << 20, h=1 << 20))
    expect(UNS, "too many", call(b=1 << 22, h=1))
    assert call(b=0) == OK and call(h=0) == OK


def test_compact_refusals():
    sh = shape()

    def call(s=sh, base=P, index=P, ss=100, sh_=50, mc=50, count=P, bt=P, k=P, v=P):
        return lib.msa_kv_compact(None if s is None else ctypes.byref(s), base, index, ss, sh_, mc, count, bt, k, v, None)
    expect(INV, "shape", call(s=None))
    expect(UNS, "head_dim", call(s=shape(head_dim=96)))
    expect(UNS, "block_size", call(s=shape(block_size=32)))
    expect(INV, "multiple", call(s=shape(num_q_heads=7)))
    bad = shape()
    bad.v_stride_dim = 12
    expect(INV, "strides", call(s=bad))
    for kw in (dict(mc=-1), dict(ss=-1), dict(sh_=-1)):
        expect(INV, ">= 0", call(**kw))
    for kw in (dict(index=None), dict(count=None), dict(bt=None), dict(k=None), dict(v=None)):
        expect(INV, "non-null", call(**kw))
    for kw in (dict(k=P + 8), dict(v=P + 8), dict(base=P + 2), dict(index=P + 2), dict(count=P + 1), dict(bt=P + 2)):
        expect(INV, "aligned", call(**kw))
    expect(UNS, "too many", call(s=shape(1 << 21)))
    assert call(s=shape(0)) == OK and call(mc=0) == OK


def test_verify_refusals():
    layout = ([500, 300], [0, 1, 2], [10, 200], [20, 100])
    plan = msa.msa_plan_tree(shape(), *layout, flags=msa.MSA_PLAN_HOST_ONLY)

    def call(h=plan.handle, kind=0, vocab=1000, ts=1000, draft=P, ds=1000):
        return lib.msa_tree_verify(h, kind, vocab, P, ts, draft, ds, P, P, P, P, P, 100, P, P, P, 1 << 20, None)
    expect(INV, "null plan", call(h=None))
    expect(INV, "prob_type", call(kind=3))
    expect(INV, "vocab", call(vocab=0))
    expect(INV, "HOST_ONLY", call())
    size = ctypes.c_size_t()
    expect(INV, "null", lib.msa_tree_verify_workspace(plan.handle, 1000, None))
    expect(INV, "vocab", lib.msa_tree_verify_workspace(plan.handle, 0, ctypes.byref(size)))
    assert msa.msa_tree_verify_workspace(plan, 1) > 0
    none = msa.msa_plan_tree(shape(), *layout, [0, 0], flags=msa.MSA_PLAN_HOST_ONLY)
    assert msa.msa_tree_verify_workspace(none, 1000) == 0


def test_tensor_checks():
    torch = pytest.importorskip("torch")
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    with pytest.raises(msa.MsaError, match="scores"):
        msa.msa_kv_select(torch.zeros(2, 3, 4), i32(2), i32(2), i32(2, 3, 4), i32(2))
    with pytest.raises(msa.MsaError, match="sequences, lists"):
        msa.msa_kv_select(torch.zeros(2, 3), i32(2), i32(2), i32(2, 3, 4), i32(2))
    with pytest.raises(msa.MsaError, match="index"):
        msa.msa_kv_compact(shape(), None, i32(2, 9), i32(2), i32(2, 200), P, P)
    plan = msa.msa_plan(shape(), [500, 300], [0, 1, 2], [10, 200], [20, 100], flags=msa.MSA_PLAN_HOST_ONLY)
    with pytest.raises(msa.MsaError, match="weights"):
        msa.msa_kv_weights(plan, P, P, P, P, torch.zeros(2, 2, 3200))
