"""From a plan of trees and causal segments to the compaction of what the verification kept, by the statements of the
read-me (GPU only)."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from tree_ref import paged  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example(holds):
    """The read-me's Python block that holds this text, with the test's sizes."""
    blocks = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md"), encoding="utf-8").read(), re.S)
    (block,) = [b for b in blocks if holds in b]
    return block.replace("num_q_heads=32, num_kv_heads=8", "num_q_heads=4, num_kv_heads=2")


def i32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# per sequence its segments (first position, parents of a tree, or a number of causal rows)
LAYOUTS = {
    "causal first": [[(0, 70)], [(37, [-1, 0, 0, 1, 2, 2, 5])]],
    "as many trees as sequences": [[(100, 9)], [(20, [-1, 0, 1, 1]), (24, [-1, 0, 0, 2, 3])]],
    "several in a block": [[(3, [-1, 0, 0]), (6, [-1, 0, 0, 2]), (10, [-1, 0, 1])], [(5, 1)], [(64, [-1] + [0] * 90)]],
    "one each": [[(5, [-1, 0, 0, 1])], [(33, [-1, 0])]],
}


@pytest.mark.parametrize("layout", LAYOUTS)
def test_kept_slots_of_every_tree_and_nothing_else(layout):
    segs = LAYOUTS[layout]
    lens = [max(s + (len(p) if isinstance(p, list) else p) for s, p in x) + 3 for x in segs]
    table, k_cache, v_cache = paged(lens, 2, 128, 1)
    MB, NB, V, layers = table.shape[1], k_cache.shape[0], 11, range(1)
    shape = msa.make_shape(len(segs), 4, 2, 128, MB, NB, 128 ** -0.5)
    flat = [(b, s, p) for b, x in enumerate(segs) for s, p in x]
    indptr = [0]
    for x in segs:
        indptr.append(indptr[-1] + len(x))
    plan = msa.msa_plan_tree(shape, lens, indptr, [s for _, s, _ in flat],
                             [len(p) if isinstance(p, list) else p for _, _, p in flat],
                             [int(isinstance(p, list)) for _, _, p in flat])
    trees = [(b, s, p) for b, s, p in flat if isinstance(p, list)]
    n = sum(len(p) for _, _, p in trees)
    assert plan.tree_rows == n
    # every last child of a node stays: its token has all of its parent's probability
    tokens, target, row, kept = torch.zeros(n, dtype=torch.int32), torch.zeros(n, V), 0, []
    for _, _, p in trees:
        children = {}
        for i, up in enumerate(p):
            if up >= 0:
                children.setdefault(up, []).append(i)
                tokens[row + i] = len(children[up]) % V
        path = [0]
        while path[-1] in children:
            last = children[path[-1]][-1]
            target[row + path[-1], tokens[row + last]] = 1.0
            first = next(i for i in children[path[-1]] if tokens[row + i] == tokens[row + last])
            path.append(first)
        target[row + path[-1], 5] = 1.0
        kept.append(path)
        row += len(p)
    path = torch.empty(len(trees), plan.max_slots, dtype=torch.int32, device="cuda")
    path_len, next_token = (torch.empty(len(trees), dtype=torch.int32, device="cuda") for _ in range(2))
    parents = i32([u for _, _, p in trees for u in p])
    ws = torch.empty(msa.msa_tree_verify_workspace(plan, V), dtype=torch.uint8, device="cuda")
    msa.msa_tree_verify(plan, target.cuda(), tokens.cuda(), parents, torch.full((n,), 0.5, device="cuda"),
                        torch.full((len(trees),), 0.5, device="cuda"), path, path_len, next_token, workspace=ws)
    assert [path[t, :path_len[t]].tolist() for t in range(len(trees))] == kept

    want_k, want_v = k_cache.clone(), v_cache.clone()
    for (b, s, _), slots in zip(trees, kept):
        for i, slot in enumerate(slots):
            src, dst = s + slot, s + i
            want_k[table[b, dst // 16].item(), :, dst % 16] = k_cache[table[b, src // 16].item(), :, src % 16]
            want_v[table[b, dst // 16].item(), :, :, dst % 16] = v_cache[table[b, src // 16].item(), :, :, src % 16]
    exec(example("tree_table"), dict(msa=msa, MB=MB, NB=NB, layers=layers, tree_seq=[b for b, _, _ in trees],
                                     tree_start=i32([s for _, s, _ in trees]), path=path, path_len=path_len,
                                     block_table=table, k_cache=k_cache, v_cache=v_cache))
    torch.cuda.synchronize()
    assert torch.equal(k_cache.view(torch.int16), want_k.view(torch.int16))
    assert torch.equal(v_cache.view(torch.int16), want_v.view(torch.int16))
