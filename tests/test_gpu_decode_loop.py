"""The tree and cache operators in the order a serving program runs them (GPU
only): a prompt with its key weights, speculative steps (mask, cache write, tree
attention, verification, compaction of the accepted slots), a reduction of the cache
(selection, compaction) and decoding on what is left, each step held against plain
64-bit forms of what the cache must then contain."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from test_gpu_cache import select64  # noqa: E402
from test_gpu_verify import walk64  # noqa: E402
from tree_ref import attention64, ancestors, random_parents  # noqa: E402

B, HQ, HKV, D, V, BLOCKS = 3, 8, 2, 128, 499, 40


class Loop:
    def __init__(self):
        g = torch.Generator().manual_seed(1)
        self.g = g
        self.shape = msa.make_shape(B, HQ, HKV, D, BLOCKS, B * BLOCKS, D ** -0.5)
        self.table = torch.randperm(B * BLOCKS, generator=g).to(torch.int32).reshape(B, BLOCKS).cuda()
        self.k = torch.zeros(B * BLOCKS, HKV, 16, D, dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros(B * BLOCKS, HKV, D, 16, dtype=torch.bfloat16, device="cuda")
        # what the caches must hold: [positions, heads, d] of each sequence
        self.keys = [torch.zeros(0, HKV, D, dtype=torch.bfloat16, device="cuda") for _ in range(B)]
        self.vals = [x.clone() for x in self.keys]
        self.weights = torch.zeros(B, HKV, BLOCKS * 16, device="cuda")
        self.head = torch.randn(HQ * D, V, generator=g).cuda() * 0.3

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g).to(torch.bfloat16).cuda()

    def lens(self):
        return [len(x) for x in self.keys]

    def cached(self, b, n):
        blk = self.table[b, :-(-n // 16)].long()
        return (self.k[blk].transpose(1, 2).reshape(-1, HKV, D)[:n], self.v[blk].permute(0, 3, 1, 2).reshape(-1, HKV, D)[:n])

    def holds_what_it_must(self):
        torch.cuda.synchronize()
        for b, n in enumerate(self.lens()):
            k, v = self.cached(b, n)
            assert torch.equal(k, self.keys[b]) and torch.equal(v, self.vals[b])

    def buffers(self, plan, rows):
        need = plan.info()["workspace_bytes"]
        return (torch.empty(rows, HQ, D, dtype=torch.bfloat16, device="cuda"), torch.empty(rows, HQ, device="cuda"),
                torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)

    def near(self, q, o, b, keys, vals, seen):
        for h in range(HQ):
            want, _, a = attention64(q[:, h], keys[:, h // (HQ // HKV)].double(), vals[:, h // (HQ // HKV)].double(),
                                     seen, D ** -0.5)
            assert ((o[:, h].double() - want).abs() <= 2.0 ** -8 * (want.abs() + a) + 1e-4).all()

    def causal(self, new):
        """new[b] rows at the end of each sequence: cache write, attention, key weights."""
        at, n = self.lens(), sum(new)
        total = [a + m for a, m in zip(at, new)]
        plan = msa.msa_plan(self.shape, total, list(range(B + 1)), at, new)
        q, k, v = self.normal(n, HQ, D), self.normal(n, HKV, D), self.normal(n, HKV, D)
        o, lse, ws = self.buffers(plan, n)
        msa.msa_kv_append(plan, k, v, self.table, self.k, self.v)
        msa.msa_forward(plan, q, self.k, self.v, self.table, o, lse, ws)
        need = msa.msa_kv_weights_workspace(plan)
        msa.msa_kv_weights(plan, q, self.k, self.table, lse, self.weights,
                           torch.empty(need, dtype=torch.uint8, device="cuda") if need else None)
        row = 0
        for b, m in enumerate(new):
            self.keys[b] = torch.cat([self.keys[b], k[row:row + m]])
            self.vals[b] = torch.cat([self.vals[b], v[row:row + m]])
            seen = torch.ones(m, total[b], dtype=torch.bool, device="cuda").tril(at[b])
            self.near(q[row:row + m], o[row:row + m], b, self.keys[b], self.vals[b], seen)
            row += m
        self.holds_what_it_must()

    def speculate(self, sizes, seed):
        r = random.Random(seed)
        parents = [random_parents(r, m, "tree") for m in sizes]
        at, n = self.lens(), sum(sizes)
        plan = msa.msa_plan_tree(self.shape, [a + m for a, m in zip(at, sizes)], list(range(B + 1)), at, sizes)
        q, k, v = self.normal(n, HQ, D), self.normal(n, HKV, D), self.normal(n, HKV, D)
        o, lse, ws = self.buffers(plan, n)
        up = torch.tensor([p for x in parents for p in x], dtype=torch.int32).cuda()
        mask = torch.empty(n, plan.mask_words, dtype=torch.int64, device="cuda")
        msa.msa_tree_mask(plan, up, mask)
        msa.msa_kv_append(plan, k, v, self.table, self.k, self.v)
        msa.msa_tree_forward(plan, q, self.k, self.v, self.table, mask, o, lse, ws)
        # the target's next-token rows, and a draft that is near them
        logits = o.reshape(n, -1).float() @ self.head
        target = torch.softmax(logits, 1)
        draft = torch.softmax(logits + 0.3 * torch.randn(n, V, generator=self.g).cuda(), 1)
        tokens, row = torch.zeros(n, dtype=torch.int32), 0
        for x in parents:
            for i, p in enumerate(x):
                if p >= 0:
                    tokens[row + i] = torch.multinomial(draft[row + p].cpu(), 1, generator=self.g)[0]
            row += len(x)
        ua, us = torch.rand(n, generator=self.g), torch.rand(B, generator=self.g)
        path = torch.empty(B, max(sizes), dtype=torch.int32, device="cuda")
        length, token = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
        ws = torch.empty(msa.msa_tree_verify_workspace(plan, V), dtype=torch.uint8, device="cuda")
        msa.msa_tree_verify(plan, target, tokens.cuda(), up, ua.cuda(), us.cuda(), path, length, token, draft, ws)
        # the accepted slots come to the front of the tree
        msa.msa_kv_compact(self.shape, torch.tensor(at, dtype=torch.int32).cuda(), path, length, self.table, self.k, self.v)
        torch.cuda.synchronize()
        row, kept = 0, 0
        for b, x in enumerate(parents):
            m = len(x)
            seen = torch.ones(m, at[b] + m, dtype=torch.bool)
            seen[:, at[b]:] = ancestors(x)
            self.near(q[row:row + m], o[row:row + m], b, torch.cat([self.keys[b], k[row:row + m]]),
                      torch.cat([self.vals[b], v[row:row + m]]), seen.cuda())
            sl = slice(row, row + m)
            want, nxt, _ = walk64(x, tokens[sl].tolist(), target[sl].double().cpu().numpy(),
                                  draft[sl].double().cpu().numpy(), ua[sl].numpy(), us[b].numpy())
            assert path[b, :length[b]].tolist() == want and int(token[b]) == nxt
            # the row of the last kept slot is the causal row of the kept tokens
            at_path = torch.tensor(want).cuda() + row
            self.keys[b] = torch.cat([self.keys[b], k[at_path]])
            self.vals[b] = torch.cat([self.vals[b], v[at_path]])
            last = at_path[-1:]
            self.near(q[last], o[last], b, self.keys[b], self.vals[b],
                      torch.ones(1, len(self.keys[b]), dtype=torch.bool, device="cuda"))
            kept += len(want)
            row += m
        self.holds_what_it_must()
        return kept

    def reduce(self, keep, first, recent):
        n = torch.tensor(self.lens(), dtype=torch.int32).cuda()
        index = torch.empty(B, HKV, max(keep), dtype=torch.int32, device="cuda")
        count = torch.empty(B, dtype=torch.int32, device="cuda")
        msa.msa_kv_select(self.weights, n, torch.tensor(keep, dtype=torch.int32).cuda(), index, count, first, recent)
        msa.msa_kv_compact(self.shape, None, index, count, self.table, self.k, self.v)
        torch.cuda.synchronize()
        for b in range(B):
            k, v = [], []
            for h in range(HKV):
                want = select64(self.weights[b, h].double().cpu().numpy(), int(n[b]), keep[b], first, recent)
                assert index[b, h, :count[b]].tolist() == want.tolist()
                at = torch.from_numpy(want).cuda()
                k.append(self.keys[b][at, h])
                v.append(self.vals[b][at, h])
                self.weights[b, h, :len(want)] = self.weights[b, h, at].clone()
                self.weights[b, h, len(want):] = 0.0
            self.keys[b], self.vals[b] = torch.stack(k, 1), torch.stack(v, 1)
        self.holds_what_it_must()


def test_prompt_speculation_reduction_and_decoding():
    s = Loop()
    s.causal([200, 37, 401])
    kept = s.speculate([9, 16, 5], 1)
    kept += s.speculate([16, 3, 12], 2)
    assert kept > 6  # more than the roots
    s.causal([1, 1, 1])
    s.reduce([100, 40, 150], 4, 16)
    s.causal([1, 30, 1])
    s.speculate([5, 5, 70], 3)
    s.reduce([64, 64, 64], 2, 8)
    s.causal([1, 1, 1])
