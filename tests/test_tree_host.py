"""Host side of msa_tree.h (no GPU): the plan's trees, refusals, declarations."""
import ctypes
import os
import re

import numpy as np
import pytest

import paper_2606_02964_amd as msa
from paper_2606_02964_amd import tree as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HOST = msa.MSA_PLAN_HOST_ONLY


def shape(num_seqs=2, **kw):
    a = dict(num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=200, num_blocks=400, scale=0.1)
    a.update(kw)
    return msa.make_shape(num_seqs, **a)


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "msa_tree.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(msa_[a-z_]+)\s*\(", text))
    assert names == set(T.EXPORTED_TREE)
    lib = ctypes.CDLL(msa.LIB_PATH)
    for n in names:
        assert hasattr(lib, n) and hasattr(msa, n)


def test_plan_figures_and_rows_are_those_of_the_causal_plan():
    layout = ([500, 300], [0, 2, 3], [10, 400, 200], [20, 70, 100])
    plan = msa.msa_plan_tree(shape(), *layout, [0, 1, 1], flags=HOST)
    assert msa.msa_plan_tree_info(plan) == {"num_trees": 2, "tree_rows": 170, "max_slots": 100, "mask_words": 2}
    same = msa.msa_plan(shape(), *layout, flags=HOST)
    assert plan.info() == same.info()
    for a, b in zip(msa.msa_plan_export(plan), msa.msa_plan_export(same)):
        assert np.array_equal(a, b)
    assert msa.msa_plan_tree_info(same) == {"num_trees": 0, "tree_rows": 0, "max_slots": 0, "mask_words": 0}
    every = msa.msa_plan_tree(shape(), *layout, flags=HOST)
    assert msa.msa_plan_tree_info(every)["num_trees"] == 3
    none = msa.msa_plan_tree(shape(0), [], [0], [], [], flags=HOST)
    assert msa.msa_plan_tree_info(none)["tree_rows"] == 0


@pytest.mark.parametrize("n,ok", [(1024, True), (1025, False)])
def test_tree_size_limit(n, ok):
    layout = ([2000], [0, 1], [100], [n])
    if ok:
        assert msa.msa_plan_tree(shape(1), *layout, flags=HOST).max_slots == n
    else:
        with pytest.raises(msa.MsaError) as e:
            msa.msa_plan_tree(shape(1), *layout, flags=HOST)
        assert e.value.status == msa.MSA_ERR_UNSUPPORTED and "1024" in str(e.value)
        msa.msa_plan_tree(shape(1), *layout, [0], flags=HOST)  # a causal segment may be longer


def test_tree_count_limit():
    n = 1 << 22
    with pytest.raises(msa.MsaError, match="trees") as e:
        msa.msa_plan_tree(shape(1, max_blocks_per_seq=n // 16), [n], [0, n], range(n), np.ones(n, dtype=np.int32),
                          flags=msa.MSA_PLAN_HOST_ONLY)
    assert e.value.status == msa.MSA_ERR_UNSUPPORTED


def test_plan_refusals():
    layout = ([500, 300], [0, 1, 2], [10, 200], [20, 100])
    for bad in ([0, 2], [-1, 1], [1]):
        with pytest.raises(msa.MsaError) as e:
            msa.msa_plan_tree(shape(), *layout, bad, flags=HOST)
        assert e.value.status == msa.MSA_ERR_INVALID_ARG and "seg_tree" in str(e.value)
    with pytest.raises(msa.MsaError) as e:
        msa.msa_plan_tree(shape(), [500, 300], [0, 1, 2], [10, 250], [20, 100], flags=HOST)
    assert e.value.status == msa.MSA_ERR_INVALID_ARG and "msa_plan_tree" in str(e.value)


def _status(fn, *args):
    return fn(*args), msa.msa_last_error()


def test_call_refusals():
    """What the library refuses before it looks at a device (addresses here are never read)."""
    lib, P = msa._lib, 4096
    layout = ([500, 300], [0, 1, 2], [10, 200], [20, 100])
    plan = msa.msa_plan_tree(shape(), *layout, flags=HOST)
    inv = msa.MSA_ERR_INVALID_ARG
    for st, text in (
            (_status(lib.msa_tree_mask, None, P, P, 2, None), "null plan"),
            (_status(lib.msa_tree_mask, plan.handle, P, P, 2, None), "HOST_ONLY"),
            (_status(lib.msa_tree_forward, None, P, P, P, P, P, 2, P, None, None, 0, None), "null plan"),
            (_status(lib.msa_tree_forward, plan.handle, P, P, P, P, P, 2, P, None, None, 0, None), "HOST_ONLY"),
            (_status(lib.msa_plan_tree_info, plan.handle, None), "null")):
        assert st[0] == inv and text in st[1], (st, text)


def test_tensor_checks():
    torch = pytest.importorskip("torch")
    plan = msa.msa_plan_tree(shape(), [500, 300], [0, 1, 2], [10, 200], [20, 100], flags=HOST)
    with pytest.raises(msa.MsaError, match="int32"):
        msa.msa_tree_mask(plan, torch.zeros(120, dtype=torch.int64), torch.zeros(120, 2, dtype=torch.int64))
    with pytest.raises(msa.MsaError, match="not on a GPU"):
        msa.msa_tree_mask(plan, torch.zeros(120, dtype=torch.int32), torch.zeros(120, 2, dtype=torch.int64))
