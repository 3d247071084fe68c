"""Tree attention, key weights, compaction and verification where element offsets
pass 2^31 (GPU only): the same small problem in the first blocks of a cache and in
blocks behind its 2^31st element, rows of probabilities likewise."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from tree_ref import random_parents  # noqa: E402


def test_blocks_behind_two_to_the_31():
    hq, hkv, d, L, m = 16, 8, 128, 300, 21
    per_block = hkv * 16 * d
    blocks = (1 << 31) // per_block + 64
    need = -(-(L + m) // 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    r = random.Random(2)
    parents = torch.tensor(random_parents(r, m, "tree"), dtype=torch.int32).cuda()
    q, qd = (torch.randn(n, hq, d, generator=g, device="cuda").bfloat16() for n in (m, L))
    k1, v1 = torch.randn(2, need, hkv, 16, d, generator=g, device="cuda").bfloat16()
    v1 = v1.transpose(2, 3).contiguous()
    k, v = (torch.empty(blocks, *x.shape[1:], dtype=torch.bfloat16, device="cuda") for x in (k1, v1))
    kept = torch.tensor([sorted(r.sample(range(L), 200))], dtype=torch.int32).cuda()
    path, count = torch.tensor([[0, 3, 9]], dtype=torch.int32).cuda(), torch.tensor([3], dtype=torch.int32).cuda()
    results = []
    for first in (0, blocks - need):
        k[first:first + need], v[first:first + need] = k1, v1
        table = torch.arange(first, first + need, dtype=torch.int32, device="cuda").flip(0)[None].contiguous()
        shape = msa.make_shape(1, hq, hkv, d, need, blocks, d ** -0.5)
        plan = msa.msa_plan_tree(shape, [L + m], [0, 1], [L], [m])
        ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
        mask = torch.empty(m, 1, dtype=torch.int64, device="cuda")
        o, lse = torch.empty_like(q), torch.empty(m, hq, device="cuda")
        msa.msa_tree_mask(plan, parents, mask)
        msa.msa_tree_forward(plan, q, k, v, table, mask, o, lse, ws)
        out = [o, lse]
        for segs in ([(0, L)], [(L - 1, 1)]):
            n = segs[0][1]
            p = msa.msa_plan(shape, [L], [0, 1], [segs[0][0]], [n])
            od, ld = torch.empty(n, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(n, hq, device="cuda")
            wb = torch.empty(max(1, p.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
            w = torch.zeros(1, hkv, need * 16, device="cuda")
            msa.msa_forward(p, qd[:n], k, v, table, od, ld, wb)
            wk = torch.empty(max(1, msa.msa_kv_weights_workspace(p)), dtype=torch.uint8, device="cuda")
            msa.msa_kv_weights(p, qd[:n], k, table, ld, w, wk)
            out.append(w)
        base = torch.tensor([L], dtype=torch.int32).cuda()
        msa.msa_kv_compact(shape, base, path, count, table, k, v)
        msa.msa_kv_compact(shape, None, kept, torch.tensor([200], dtype=torch.int32).cuda(), table, k, v)
        torch.cuda.synchronize()
        out += [k[first:first + need].clone(), v[first:first + need].clone()]
        results.append(out)
    for a, b in zip(*results):
        assert torch.equal(a.view(torch.int16 if a.dtype == torch.bfloat16 else torch.int32),
                           b.view(torch.int16 if b.dtype == torch.bfloat16 else torch.int32))
    assert not torch.equal(results[0][5], k1)  # something moved


@pytest.mark.parametrize("vocab", [30011, 70001])
def test_rows_behind_two_to_the_31(vocab):
    """The last trees of a batch whose rows pass 2^31 elements give what they give alone."""
    slots = 64
    trees = (1 << 31) // (slots * vocab) + 2
    r = random.Random(3)
    parents = torch.tensor(random_parents(r, slots, "tree"), dtype=torch.int32).cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    rows = trees * slots
    target = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    draft = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")
    last = slice(rows - 2 * slots, rows)
    logits = 3 * torch.randn(2 * slots, vocab, generator=g, device="cuda")
    target[last] = torch.softmax(logits, 1).bfloat16()
    draft[last] = torch.softmax(logits + 0.7 * torch.randn(2 * slots, vocab, generator=g, device="cuda"), 1).bfloat16()
    tokens = torch.multinomial(draft[last].float(), slots, replacement=True, generator=g)
    up = parents.repeat(2).long().clamp(min=0) + torch.arange(2, device="cuda").repeat_interleave(slots) * slots
    tok = tokens[up, torch.arange(slots, device="cuda").repeat(2)].to(torch.int32)
    ua, us = torch.rand(2 * slots, generator=g, device="cuda"), torch.rand(2, generator=g, device="cuda")

    def run(n, target, draft):
        m = [slots] * n
        shape = msa.make_shape(n, 8, 8, 128, slots // 16, n * slots // 16, 1.0)
        plan = msa.msa_plan_tree(shape, m, list(range(n + 1)), [0] * n, m)
        t, a, s = torch.zeros(n * slots, dtype=torch.int32, device="cuda"), torch.zeros(n * slots, device="cuda"), torch.zeros(n, device="cuda")
        t[-2 * slots:], a[-2 * slots:], s[-2:] = tok, ua, us
        path = torch.empty(n, slots, dtype=torch.int32, device="cuda")
        length, nxt = torch.empty(n, dtype=torch.int32, device="cuda"), torch.empty(n, dtype=torch.int32, device="cuda")
        ws = torch.empty(msa.msa_tree_verify_workspace(plan, vocab), dtype=torch.uint8, device="cuda")
        msa.msa_tree_verify(plan, target, t, parents.repeat(n), a, s, path, length, nxt, draft, ws)
        torch.cuda.synchronize()
        return path[-2:], length[-2:], nxt[-2:], length, nxt

    alone = run(2, target[last].clone(), draft[last].clone())
    far = run(trees, target, draft)
    assert all(torch.equal(a, b) for a, b in zip(alone[:3], far[:3]))
    assert (far[3][:-2] == 1).all() and (far[4][:-2] == -1).all()  # rows of zeros: nothing to draw from
