"""Attention of trees of drafted tokens (msa_tree_mask, msa_tree_forward)
against a plain 64-bit implementation (GPU only).

The output's bar, element by element: half a bf16 step of the output and half a
bf16 step of every weight, 2^-8 (|o| + sum_j p_j |v_j|), plus 1e-4 for the fp32
sums (128 products of a score: 128 * 2^-24 * sum |q k| * scale < 1e-4).  The
lse's: 2e-4, the same score error and that of the fp32 exponentials and sums.
"""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from tree_ref import ancestors, attention64, mask_words, paged, random_parents, rows64  # noqa: E402

HEADS = {"d128": (8, 2, 128), "d64": (4, 4, 64), "wide": (16, 2, 128), "mqa": (20, 1, 64)}


class Step:
    """One step's inputs.  segs: per sequence a list of (start, length, parents or None for a causal segment)."""

    def __init__(self, segs, heads=(8, 2, 128), seed=1, q_pad=0, seen=None, flags=0, split=0, stride_more=0):
        self.segs, self.hq, self.hkv, self.d = segs, *heads
        self.lens = [max((s + n for s, n, _ in x), default=0) for x in segs]
        self.table, self.k, self.v = paged(self.lens, self.hkv, self.d, seed)
        g = torch.Generator().manual_seed(seed + 1)
        self.rows = sum(n for x in segs for _, n, _ in x)
        width = self.hq * self.d + q_pad
        self.q = torch.randn(self.rows + 2, width, generator=g).to(torch.bfloat16).cuda()
        self.scale = self.d ** -0.5
        flat = [y for x in segs for y in x]
        self.trees = [p for _, _, p in flat if p is not None]
        self.parents = torch.tensor([x for p in self.trees for x in p], dtype=torch.int32).cuda()
        self.seen = seen if seen is not None else [ancestors(p) for p in self.trees]
        self.shape = msa.make_shape(len(segs), self.hq, self.hkv, self.d, self.table.shape[1], self.k.shape[0],
                                    self.scale, q_strides=(width, self.d), o_strides=(width, self.d))
        indptr = [0]
        for x in segs:
            indptr.append(indptr[-1] + len(x))
        self.layout = (self.lens, indptr, [s for s, _, _ in flat], [n for _, n, _ in flat])
        self.plan = msa.msa_plan_tree(self.shape, *self.layout, [int(p is not None) for _, _, p in flat],
                                      flags=flags, kv_split_tokens=split)
        self.words = max(1, self.plan.mask_words)
        mask = torch.full((self.plan.tree_rows, self.words + stride_more), -1, dtype=torch.int64)
        at = 0
        for s in self.seen:
            mask[at:at + len(s), :self.words] = mask_words(s, self.words)
            at += len(s)
        self.mask = mask.cuda()
        self.o = torch.full((self.rows + 2, width), 7.0, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.full((self.rows + 2, self.hq), 7.0, device="cuda")
        need = self.plan.info()["workspace_bytes"]
        self.ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda") if need else None

    def forward(self, stream=None, lse=True):
        msa.msa_tree_forward(self.plan, self.q, self.k, self.v, self.table, self.mask, self.o,
                             self.lse if lse else None, self.ws, stream=stream)

    def reference(self):
        G, row, tree = self.hq // self.hkv, 0, 0
        o = torch.zeros(self.rows, self.hq, self.d, dtype=torch.float64, device="cuda")
        a, lse = torch.zeros_like(o), torch.zeros(self.rows, self.hq, dtype=torch.float64, device="cuda")
        q = self.q[:, :self.hq * self.d].reshape(-1, self.hq, self.d)
        for b, x in enumerate(self.segs):
            for s, n, p in x:
                seen = torch.ones(n, s + n, dtype=torch.bool)
                seen[:, s:] = torch.ones(n, n, dtype=torch.bool).tril()
                if p is not None:
                    seen[:, s:] &= self.seen[tree]
                    tree += 1
                seen = seen.cuda()
                for h in range(self.hq):
                    k = rows64(self.k, self.table[b], s + n, h // G, False)
                    v = rows64(self.v, self.table[b], s + n, h // G, True)
                    o[row:row + n, h], lse[row:row + n, h], a[row:row + n, h] = attention64(
                        q[row:row + n, h], k, v, seen, self.scale)
                row += n
        return o, lse, a

    def check(self, lse=True):
        torch.cuda.synchronize()
        o, l, a = self.reference()
        n = self.hq * self.d
        got = self.o[:self.rows, :n].reshape(o.shape).double()
        assert torch.isfinite(got).all()
        err = (got - o).abs() - 2.0 ** -8 * (o.abs() + a) - 1e-4
        assert (err <= 0).all(), err.max().item()
        if lse:
            hidden = l == -float("inf")
            assert torch.equal(self.lse[:self.rows].double() == -float("inf"), hidden)
            assert (self.lse[:self.rows].double() - l)[~hidden].abs().max().item() <= 2e-4 if (~hidden).any() else True
            assert (got[hidden] == 0).all()
        # rows behind the last one, and what lies between rows, stay as they were
        assert (self.o[self.rows:] == 7).all() and (self.o[:, n:] == 7).all() and (self.lse[self.rows:] == 7).all()


def tree(r, ctx, m, kind="tree"):
    return (ctx, m, random_parents(r, m, kind))


@pytest.mark.parametrize("kind", ["tree", "chain", "star", "forest"])
@pytest.mark.parametrize("heads", list(HEADS))
def test_small_trees_at_block_and_step_borders(kind, heads):
    r = random.Random(5)
    ctxs = [0, 1, 15, 16, 17, 47, 63, 64, 65, 127, 200]
    s = Step([[tree(r, c, 1 + (7 * i + 3) % 13, kind)] for i, c in enumerate(ctxs)], HEADS[heads])
    s.forward()
    s.check()


@pytest.mark.parametrize("m", [1, 2, 16, 17, 63, 64, 65, 128, 130, 200, 1024])
@pytest.mark.parametrize("ctx", [0, 37, 700])
def test_tree_sizes(m, ctx):
    r = random.Random(m)
    s = Step([[tree(r, ctx, m)], [tree(r, ctx + 5, max(1, m // 2), "chain")]], HEADS["d128"], stride_more=1)
    s.forward()
    s.check()


@pytest.mark.parametrize("flags", [0, msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128,
                                   msa.MSA_PLAN_TILE_ROWS_256, msa.MSA_PLAN_PRECISE_WEIGHTS,
                                   msa.MSA_PLAN_PRECISE_WEIGHTS | msa.MSA_PLAN_TILE_ROWS_32])
@pytest.mark.parametrize("split", [0, 64, 256])
@pytest.mark.parametrize("heads", ["d128", "d64"])
def test_every_kernel_and_split(flags, split, heads):
    r = random.Random(9)
    s = Step([[tree(r, 1000, 61)], [tree(r, 333, 24), (400, 50, None)], [(100, 70, None), tree(r, 180, 100)],
              [], [tree(r, 2111, 7)]], HEADS[heads], flags=flags, split=split, q_pad=16)
    s.forward()
    s.check()


@pytest.mark.parametrize("ctx,slots,heads", [(8190, 61, (32, 8, 128)), (3000, 40, (16, 2, 128)), (5000, 100, (4, 4, 64))])
def test_one_long_sequence(ctx, slots, heads):
    """A small plan, cut to a piece per CU."""
    s = Step([[tree(random.Random(1), ctx, slots)]], heads)
    assert s.plan.info()["num_merge"] > 0 and s.plan.info()["num_workgroups"] <= 256
    s.forward()
    s.check()


def test_many_workgroups():
    """More tiles than CUs: the 128-row kernel without helpers, several items a workgroup."""
    r = random.Random(2)
    s = Step([[tree(r, 300 + 41 * i, 40)] for i in range(24)], (32, 16, 128))
    s.forward()
    s.check()


@pytest.mark.parametrize("flags", [msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128,
                                   msa.MSA_PLAN_TILE_ROWS_256])
@pytest.mark.parametrize("split", [0, 64])
def test_any_mask_and_rows_that_see_nothing(flags, split):
    """Random bits, also of later slots (never used); without context, a row whose mask is empty sees nothing."""
    g = torch.Generator().manual_seed(3)
    sizes = [(0, 40), (0, 1), (0, 150), (70, 90)]
    seen = [torch.rand(m, m, generator=g) < 0.3 for _, m in sizes]
    for x in seen[:3]:
        x[::3] = False
    s = Step([[(c, m, [-1] * m)] for c, m in sizes], HEADS["d64"], seen=seen, flags=flags, split=split)
    s.forward()
    s.check()
    assert torch.isinf(s.lse[:s.rows]).any()


@pytest.mark.parametrize("flags", [0, msa.MSA_PLAN_TILE_ROWS_128])
def test_hidden_keys_may_hold_anything(flags):
    """K of slots that no row but their own sees holds NaN and infinities: every other row is as without."""
    star = [-1] + [0] * 30
    s = Step([[(50, 31, star)]], flags=flags)
    seen = [torch.zeros(31, 31, dtype=torch.bool)]
    seen[0][:, 0] = True
    for i in range(0, 31, 2):
        seen[0][i, i] = True
    s = Step([[(50, 31, star)]], seen=seen, flags=flags)
    for j in range(1, 31, 2):
        pos = 50 + j
        s.k[s.table[0, pos // 16].long(), :, pos % 16] = float("nan") if j % 4 == 1 else float("inf")
    s.forward()
    s.check()


def test_a_chain_is_the_causal_call():
    s = Step([[(129, 40, list(range(-1, 39)))], [(5, 3, [-1, 0, 1])]])
    s.forward()
    plan = msa.msa_plan(s.shape, *s.layout)
    o, lse = torch.empty_like(s.o), torch.empty_like(s.lse)
    msa.msa_forward(plan, s.q, s.k, s.v, s.table, o, lse, s.ws)
    s.check()
    n, hd = s.rows, s.hq * s.d
    assert (s.lse[:n] - lse[:n]).abs().max().item() <= 1e-5
    assert (s.o[:n, :hd].float() - o[:n, :hd].float()).abs().max().item() <= 2.0 ** -6  # a step of a value below 4


def test_masks_from_parents():
    r = random.Random(11)
    segs = [[tree(r, 3, 1)], [(0, 9, None), tree(r, 20, 64), tree(r, 100, 65, "chain")], [tree(r, 0, 1024)],
            [tree(r, 7, 300, "forest")]]
    s = Step(segs, stride_more=2)
    parents = s.parents.clone()
    parents[0] = 5        # outside [0, own slot): no parent
    parents[1] = 1 << 30
    mask = torch.full_like(s.mask, -7)
    msa.msa_tree_mask(s.plan, parents, mask)
    torch.cuda.synchronize()
    assert torch.equal(mask[:, :s.words], s.mask[:, :s.words])
    assert (mask[:, s.words:] == -7).all()


def test_plan_with_causal_segments_only_and_with_no_rows():
    s = Step([[(10, 90, None)], [(0, 1, None)]])
    msa.msa_tree_forward(s.plan, s.q, s.k, s.v, s.table, None, s.o, s.lse, s.ws)
    s.check()
    empty = Step([[], []])
    empty.forward()
    msa.msa_tree_mask(empty.plan, empty.parents, empty.mask)
    empty.check()


def test_deterministic_and_without_lse():
    r = random.Random(4)
    s = Step([[tree(r, 900, 33)], [tree(r, 4000, 12)]])
    s.forward()
    a, l = s.o.clone(), s.lse.clone()
    s.o.fill_(7.0)
    s.forward(lse=False)
    torch.cuda.synchronize()
    assert torch.equal(a.view(torch.int16), s.o.view(torch.int16)) and torch.equal(l, s.lse)


def test_step_in_a_graph_and_on_another_stream():
    """Mask, cache write and attention captured together; every replay equals the eager step on the same inputs."""
    r = random.Random(8)
    s = Step([[tree(r, 515, 20)], [tree(r, 90, 31)]])
    g = torch.Generator().manual_seed(1)
    kv = torch.randn(s.rows, 2 * s.hkv, s.d, generator=g).to(torch.bfloat16).cuda()

    def step(stream=None):
        msa.msa_tree_mask(s.plan, s.parents, s.mask, stream=stream)
        msa.msa_kv_append(s.plan, kv[:, :s.hkv], kv[:, s.hkv:], s.table, s.k, s.v, stream=stream)
        s.forward(stream)

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    step(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        kv.normal_()
        s.q.normal_()
        s.mask.zero_()
        graph.replay()
        torch.cuda.synchronize()
        s.check()
        got = s.o.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got.view(torch.int16), s.o.view(torch.int16))
