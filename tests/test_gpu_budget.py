"""A cache within a budget over several reductions, by the statements of the read-me: every key's sum has to be the
sum of the weights that this very key received, wherever compaction has put it (GPU only).

The bar is that of test_gpu_cache.py, 2^-17 of the sum plus 2^-20 of it for each call that added to it."""
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from test_gpu_cache import select64  # noqa: E402
from test_gpu_tree_commit import example, i32  # noqa: E402

B, HQ, HKV, D, MB = 3, 4, 2, 64, 20


class Budget:
    def __init__(self):
        self.g = torch.Generator().manual_seed(5)
        self.shape = msa.make_shape(B, HQ, HKV, D, MB, B * MB, D ** -0.5)
        self.table = torch.randperm(B * MB, generator=self.g).to(torch.int32).reshape(B, MB).cuda()
        self.k = torch.zeros(B * MB, HKV, 16, D, dtype=torch.bfloat16, device="cuda")
        self.v = torch.zeros(B * MB, HKV, D, 16, dtype=torch.bfloat16, device="cuda")
        self.weights = torch.zeros(B, HKV, MB * 16, device="cuda")
        self.keys = [[torch.zeros(0, D, dtype=torch.float64)] * HKV for _ in range(B)]
        self.sums = [[torch.zeros(0, dtype=torch.float64)] * HKV for _ in range(B)]
        self.calls = 0

    def normal(self, *s):
        return torch.randn(*s, generator=self.g).to(torch.bfloat16).cuda()

    def step(self, new):
        at, n = [len(x[0]) for x in self.keys], sum(new)
        plan = msa.msa_plan(self.shape, [a + m for a, m in zip(at, new)], list(range(B + 1)), at, new)
        q, k, v = self.normal(n, HQ, D), self.normal(n, HKV, D), self.normal(n, HKV, D)
        o, lse = torch.empty_like(q), torch.empty(n, HQ, device="cuda")
        ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
        msa.msa_kv_append(plan, k, v, self.table, self.k, self.v)
        msa.msa_forward(plan, q, self.k, self.v, self.table, o, lse, ws)
        exec(example("msa_kv_weights(plan"), dict(msa=msa, torch=torch, plan=plan, layers=range(1), q=q, k_cache=self.k,
                                              block_table=self.table, lse=lse, weights=self.weights))
        torch.cuda.synchronize()
        self.calls += 1
        q, k, lse, row, G = q.cpu().double(), k.cpu().double(), lse.cpu().double(), 0, HQ // HKV
        for b, m in enumerate(new):
            seen = torch.ones(m, at[b] + m, dtype=torch.bool).tril(at[b])
            for h in range(HKV):
                self.keys[b][h] = torch.cat([self.keys[b][h], k[row:row + m, h]])
                w = torch.zeros(at[b] + m, dtype=torch.float64)
                for i in range(h * G, h * G + G):
                    s = q[row:row + m, i] @ self.keys[b][h].T * D ** -0.5 - lse[row:row + m, i, None]
                    w += torch.where(seen, torch.exp(s), 0.0).sum(0)
                self.sums[b][h] = torch.cat([self.sums[b][h], torch.zeros(m, dtype=torch.float64)]) + w
            row += m
        self.holds()

    def holds(self):
        for b in range(B):
            for h in range(HKV):
                n, want = len(self.sums[b][h]), self.sums[b][h]
                got = self.weights[b, h].cpu().double()
                assert ((got[:n] - want).abs() <= (2.0 ** -17 + self.calls * 2.0 ** -20) * want).all(), (b, h)
                assert (got[n:] == 0.0).all()

    def reduce(self, keep):
        lens = [len(x[0]) for x in self.keys]
        scores = self.weights.cpu().double().numpy()
        index = torch.full((B, HKV, max(keep)), 1 << 30, dtype=torch.int32, device="cuda")
        count = torch.empty(B, dtype=torch.int32, device="cuda")
        exec(example("msa_kv_select("), dict(msa=msa, torch=torch, shape=self.shape, layers=range(1), weights=self.weights,
                                             seq_len=i32(lens), keep=i32(keep), index=index, count=count,
                                             block_table=self.table, k_cache=self.k, v_cache=self.v))
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(HKV):
                at = torch.from_numpy(select64(scores[b, h], lens[b], keep[b], 4, 64))
                assert len(at) == int(count[b])
                self.keys[b][h], self.sums[b][h] = self.keys[b][h][at], self.sums[b][h][at]
        self.holds()


def test_every_sum_stays_with_its_key():
    s = Budget()
    s.step([200, 90, 150])
    s.step([1, 1, 1])
    s.reduce([100, 300, 80])  # the second sequence keeps all it has
    for new in ([1, 1, 1], [5, 40, 1]):
        s.step(new)
    s.reduce([70, 75, 72])
    for new in ([1, 1, 1], [30, 1, 3], [1, 1, 1]):
        s.step(new)
    s.reduce([90, 66, 20])
    s.step([1, 1, 1])
