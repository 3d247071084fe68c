"""What the binding of msa_tree.h and msa_cache.h refuses of tensors before the library sees an address (no GPU; the
addresses given are never read: every call is refused)."""
import pytest

import paper_2606_02964_amd as msa

torch = pytest.importorskip("torch")

P = 4096  # an address
SHAPE = msa.make_shape(2, 8, 2, 128, 40, 80, 0.1)
LAYOUT = ([500, 300], [0, 1, 2], [10, 200], [20, 100])


def zeros(*s, dtype=torch.int32):
    return torch.zeros(*s, dtype=dtype)


@pytest.fixture(scope="module")
def plan():
    return msa.msa_plan(SHAPE, *LAYOUT, flags=msa.MSA_PLAN_HOST_ONLY)


@pytest.fixture(scope="module")
def trees():
    return msa.msa_plan_tree(SHAPE, *LAYOUT, flags=msa.MSA_PLAN_HOST_ONLY)


def refused(match, call, **kw):
    with pytest.raises(msa.MsaError, match=match) as e:
        call(**kw)
    assert e.value.status == msa.MSA_ERR_INVALID_ARG


# (argument, a tensor of a wrong type, a tensor of the right type that is on the host)
VALUES = [zeros(9, dtype=torch.float16), zeros(9, dtype=torch.float32), zeros(9, dtype=torch.int64)]
TABLES = [zeros(2, 40, dtype=torch.int64), zeros(2, 40, dtype=torch.int16), zeros(2, 40, dtype=torch.float32)]
LSES = [zeros(120, 8, dtype=t) for t in (torch.bfloat16, torch.float16, torch.float64)]


def test_tree_forward(trees):
    def call(q=P, k_cache=P, v_cache=P, block_table=P, mask=P, o=P, lse=P, workspace=None, **kw):
        msa.msa_tree_forward(trees, q, k_cache, v_cache, block_table, mask, o, lse, workspace, **kw)
    for name in ("q", "k_cache", "v_cache", "o"):
        for x in VALUES:
            refused(f"{name} has type", call, **{name: x})
        refused(f"{name} is not on a GPU", call, **{name: zeros(9, dtype=torch.bfloat16)})
    for x in TABLES:
        refused("block_table has type", call, block_table=x)
    refused("block_table is not on a GPU", call, block_table=zeros(2, 40))
    for x in LSES:
        refused("lse has type", call, lse=x)
    refused("lse is not on a GPU", call, lse=zeros(120, 8, dtype=torch.float32))
    refused("mask has type", call, mask=zeros(120, 2))
    refused("workspace is not on a GPU", call, workspace=zeros(64, dtype=torch.uint8))
    refused("workspace_bytes", call, workspace=P)
    refused("HOST_ONLY", call)  # all of it passed on to the library
    refused("HOST_ONLY", call, workspace=P, workspace_bytes=64)
    refused("HOST_ONLY", call, lse=None)


def test_weights(plan):
    def call(q=P, k_cache=P, block_table=P, lse=P, weights=zeros(2, 2, 640, dtype=torch.float32), **kw):
        msa.msa_kv_weights(plan, q, k_cache, block_table, lse, weights, **kw)
    refused("weights is not on a GPU", call)
    refused("weights is not a tensor", call, weights=P)
    refused("weights is not a tensor", call, weights=zeros(2, 640, dtype=torch.float32))
    refused("weights has type", call, weights=zeros(2, 2, 640, dtype=torch.bfloat16))


def test_compact():
    def call(base=P, index=zeros(2, 9), count=P, block_table=P, k_cache=P, v_cache=P):
        msa.msa_kv_compact(SHAPE, base, index, count, block_table, k_cache, v_cache)
    refused("index is not on a GPU", call)
    refused("index has type", call, index=zeros(2, 9, dtype=torch.int64))
    refused("index is not on a GPU", call, index=zeros(2, 2, 9))
    refused("index is not a tensor", call, index=zeros(18))
    refused("index is not a tensor", call, index=P)


def test_verify(trees):
    def call(target=zeros(120, 50, dtype=torch.float32), **kw):
        msa.msa_tree_verify(trees, target, P, P, P, P, P, P, P, **kw)
    refused("target is not on a GPU", call)
    refused("target is not a 2-D", call, target=P)
    refused("target is not a 2-D", call, target=None)
    refused("target has type", call, target=zeros(120, 50, dtype=torch.float64))


def test_mask_strides(trees):
    refused("mask is not on a GPU", msa.msa_tree_mask, plan=trees, parents=P, mask=zeros(120, 2, dtype=torch.int64))
    refused("parents has type", msa.msa_tree_mask, plan=trees, parents=zeros(120, dtype=torch.int64), mask=P)
    refused("HOST_ONLY", msa.msa_tree_mask, plan=trees, parents=P, mask=P)


class OnDevice:
    """What the checks ask of a tensor, on any device."""
    is_cuda = True

    def __init__(self, *shape, dtype=torch.int32, device=0, strides=None):
        self.shape, self.dtype, self._device = tuple(shape), dtype, device
        self._strides = strides or torch.zeros(0).new_empty(shape, device="meta").stride()

    def stride(self, i=None):
        return self._strides if i is None else self._strides[i]

    def dim(self):
        return len(self.shape)

    def numel(self):
        return torch.Size(self.shape).numel()

    def element_size(self):
        return torch.empty(0, dtype=self.dtype).element_size()

    def get_device(self):
        return self._device

    def is_contiguous(self):
        return self._strides == torch.empty(self.shape, device="meta").stride()

    def data_ptr(self):
        return P


@pytest.fixture
def device0(monkeypatch):
    monkeypatch.setattr("paper_2606_02964_amd.tree._device", lambda: 0)
    monkeypatch.setattr("paper_2606_02964_amd.tree._raw_stream", lambda dev: None)


F32, BF16 = torch.float32, torch.bfloat16


def args(plan_kind, **kw):
    if plan_kind == "weights":
        a = dict(q=OnDevice(120, 8, 128, dtype=BF16), k_cache=OnDevice(80, 2, 16, 128, dtype=BF16),
                 block_table=OnDevice(2, 40), lse=OnDevice(120, 8, dtype=F32), weights=OnDevice(2, 2, 640, dtype=F32),
                 workspace=OnDevice(64, dtype=torch.uint8))
    elif plan_kind == "forward":
        a = dict(q=OnDevice(120, 8, 128, dtype=BF16), k_cache=OnDevice(80, 2, 16, 128, dtype=BF16),
                 v_cache=OnDevice(80, 2, 128, 16, dtype=BF16), block_table=OnDevice(2, 40),
                 mask=OnDevice(120, 2, dtype=torch.int64), o=OnDevice(120, 8, 128, dtype=BF16),
                 lse=OnDevice(120, 8, dtype=F32), workspace=OnDevice(64, dtype=torch.uint8))
    elif plan_kind == "compact":
        a = dict(base=OnDevice(2), index=OnDevice(2, 0), count=OnDevice(2), block_table=OnDevice(2, 40),
                 k_cache=OnDevice(80, 2, 16, 128, dtype=BF16), v_cache=OnDevice(80, 2, 128, 16, dtype=BF16))
    elif plan_kind == "select":
        a = dict(scores=OnDevice(2, 0, 640, dtype=F32), index=OnDevice(2, 0, 64), seq_len=OnDevice(2), keep=OnDevice(2),
                 count=OnDevice(2))
    else:
        a = dict(target=OnDevice(120, 50, dtype=F32), draft=OnDevice(120, 50, dtype=F32), tokens=OnDevice(120),
                 parents=OnDevice(120), u_accept=OnDevice(120, dtype=F32), u_sample=OnDevice(2, dtype=F32),
                 path=OnDevice(2, 100), path_len=OnDevice(2), next_token=OnDevice(2),
                 workspace=OnDevice(1 << 16, dtype=torch.uint8))
    a.update(kw)
    return a


def calls(plan, trees):
    return {"weights": (lambda **a: msa.msa_kv_weights(plan, **a)), "forward": (lambda **a: msa.msa_tree_forward(trees, **a)),
            "compact": (lambda **a: msa.msa_kv_compact(SHAPE, **a)), "select": (lambda **a: msa.msa_kv_select(**a)),
            "verify": (lambda **a: msa.msa_tree_verify(trees, **a))}


# Calls that reach the library do nothing there: the plans are host-only, compaction's and selection's lists empty.
REACHED = {"weights": "HOST_ONLY", "forward": "HOST_ONLY", "verify": "HOST_ONLY", "compact": None, "select": None}


@pytest.mark.parametrize("kind", REACHED)
def test_tensors_of_another_device(device0, plan, trees, kind):
    call = calls(plan, trees)[kind]
    if REACHED[kind]:
        refused(REACHED[kind], call, **args(kind))
    else:
        call(**args(kind))
    for name, x in args(kind).items():
        x._device = 1
        refused(f"{name} is on device 1, the current device is 0", call, **args(kind, **{name: x}))


SHORT = {
    "weights": dict(block_table=OnDevice(2, 39), lse=OnDevice(119, 8, dtype=F32), weights=OnDevice(2, 2, 639, dtype=F32)),
    "forward": dict(block_table=OnDevice(1, 40), lse=OnDevice(120, 7, dtype=F32), mask=OnDevice(120, 1, dtype=torch.int64)),
    "compact": dict(base=OnDevice(1), count=OnDevice(1), block_table=OnDevice(79), index=OnDevice(1, 0)),
    "select": dict(seq_len=OnDevice(1), keep=OnDevice(0), count=OnDevice(1), index=OnDevice(1, 0, 64)),
    "verify": dict(target=OnDevice(119, 50, dtype=F32), draft=OnDevice(120, 49, dtype=F32), tokens=OnDevice(119),
                   parents=OnDevice(119), u_accept=OnDevice(119, dtype=F32), u_sample=OnDevice(1, dtype=F32),
                   path=OnDevice(2, 99), path_len=OnDevice(1), next_token=OnDevice(1)),
}


@pytest.mark.parametrize("kind", SHORT)
def test_short_and_strided_tensors(device0, plan, trees, kind):
    call = calls(plan, trees)[kind]
    for name, x in SHORT[kind].items():
        refused(f"{name} has .* needed", call, **args(kind, **{name: x}))
    for name in ("block_table", "lse", "tokens", "count"):
        x = args(kind).get(name)
        if x is not None:
            x._strides = tuple(2 * s for s in x._strides)
            refused(f"{name} is not contiguous", call, **args(kind, **{name: x}))


@pytest.mark.parametrize("kind", REACHED)
def test_types(device0, plan, trees, kind):
    call = calls(plan, trees)[kind]
    for name, x in args(kind).items():
        if name == "workspace":
            continue
        x.dtype = torch.float64 if x.dtype != torch.float64 else torch.int32
        refused(f"{name} has type", call, **args(kind, **{name: x}))
        x.dtype = torch.int64
        if name != "mask":
            refused(f"{name} has type", call, **args(kind, **{name: x}))


def test_a_row_stride_other_than_the_tensors(device0, trees):
    mask = OnDevice(120, 3, dtype=torch.int64)
    refused("3 elements from row to row, not 100", msa.msa_tree_mask, plan=trees, parents=OnDevice(120), mask=mask, mask_stride=100)
    refused("HOST_ONLY", msa.msa_tree_mask, plan=trees, parents=OnDevice(120), mask=mask, mask_stride=3)
    refused("HOST_ONLY", msa.msa_tree_mask, plan=trees, parents=OnDevice(120), mask=P, mask_stride=100)


@pytest.mark.parametrize("size", [1 << 31, (1 << 32) + 5, 1 << 40])
def test_sizes_that_do_not_fit_the_librarys_arguments(device0, plan, trees, size):
    call = calls(plan, trees)
    refused(f"first {size}", call["select"], **args("select", first=size))
    refused(f"recent {size}", call["select"], **args("select", recent=size))
    refused("recent -2147483649", call["select"], **args("select", recent=-(1 << 31) - 1))
    refused("sizes", call["select"], **args("select", recent=-1))
    refused(f"positions {size}", call["select"], **args("select", scores=OnDevice(2, 0, size, dtype=F32)))
    refused(f"entries {size}", call["select"], **args("select", index=OnDevice(2, 0, size)))
    refused(f"entries {size}", call["compact"], **args("compact", index=OnDevice(2, size)))
    refused(f"entries {size}", call["compact"], **args("compact", index=OnDevice(2, 2, size)))
    wide = OnDevice(120, size, dtype=F32)
    refused(f"vocab {size}", call["verify"], **args("verify", target=wide, draft=wide))
    refused(f"vocab {size}", msa.msa_tree_verify_workspace, plan=trees, vocab=size)


def test_a_closed_plan(device0):
    for make, call in ((msa.msa_plan, "weights"), (msa.msa_plan_tree, "forward"), (msa.msa_plan_tree, "verify")):
        p = make(SHAPE, *LAYOUT, flags=msa.MSA_PLAN_HOST_ONLY)
        p.close()
        a = {"weights": (P, P, P, P, OnDevice(2, 2, 640, dtype=F32)), "forward": (P, P, P, P, P, P),
             "verify": (OnDevice(120, 50, dtype=F32), P, P, P, P, P, P, P)}[call]
        fn = {"weights": msa.msa_kv_weights, "forward": msa.msa_tree_forward, "verify": msa.msa_tree_verify}[call]
        with pytest.raises(msa.MsaError, match="null plan"):
            fn(p, *a)
