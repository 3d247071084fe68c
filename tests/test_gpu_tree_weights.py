"""Key weights of a speculative step: only the slots that the verification kept give weight, by the statements of the
read-me (GPU only).

The bar is that of test_gpu_cache.py, 2^-17 of a key's weight, plus 2^-20 of what stood there before."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from test_gpu_tree_commit import example, i32  # noqa: E402
from tree_ref import paged, random_parents, rows64  # noqa: E402


@pytest.mark.parametrize("sizes", [[1, 2, 3], [9, 16, 5], [70, 33, 64]])
@pytest.mark.parametrize("kind", ["chain", "tree", "star"])
def test_rows_that_stay_give_weight(kind, sizes):
    r, g = random.Random(3), torch.Generator().manual_seed(4)
    B, HQ, HKV, D, V = 3, 8, 2, 128, 23
    at = [200, 37, 512]
    parents = [random_parents(r, m, kind) for m in sizes]
    n = sum(sizes)
    seq_kv_len = [a + m for a, m in zip(at, sizes)]
    table, k_cache, v_cache = paged(seq_kv_len, HKV, D, 2)
    shape = msa.make_shape(B, HQ, HKV, D, table.shape[1], k_cache.shape[0], D ** -0.5)
    normal = lambda *s: torch.randn(*s, generator=g).to(torch.bfloat16).cuda()  # noqa: E731
    # even slots' tokens always stay, odd ones' hardly ever
    tokens = torch.arange(n, dtype=torch.int32) % 2
    target = torch.full((n, V), 0.5 / (V - 1))
    target[:, 0] = 0.5
    draft = torch.full((n, V), 1.0 / V)
    draft[:, 0], draft[:, 1] = 0.01, 0.9
    names = dict(
        msa=msa, torch=torch, layers=range(1), shape=shape, seq_kv_len=seq_kv_len, seg_indptr=list(range(B + 1)),
        seg_start=at, seg_len=sizes, parents=i32([p for x in parents for p in x]), q=normal(n, HQ, D),
        k_new=normal(n, HKV, D), v_new=normal(n, HKV, D), block_table=table, k_cache=k_cache, v_cache=v_cache,
        o=torch.empty(n, HQ, D, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(n, HQ, device="cuda"),
        ws=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"), vocab=V, target=target.cuda(), draft=draft.cuda(),
        tokens=tokens.cuda(), u_accept=torch.rand(n, generator=g).cuda(), u_sample=torch.rand(B, generator=g).cuda(),
        path=torch.empty(B, max(sizes), dtype=torch.int32, device="cuda"),
        path_len=torch.empty(B, dtype=torch.int32, device="cuda"),
        next_token=torch.empty(B, dtype=torch.int32, device="cuda"), tree_start=i32(at))
    exec(example("msa_tree_verify("), names)
    torch.cuda.synchronize()
    before = torch.rand(B, HKV, table.shape[1] * 16, generator=g).cuda()
    names["weights"] = before.clone()
    row_of = [sum(sizes[:b]) for b in range(B)]
    names["tree_of"] = torch.tensor([b for b, m in enumerate(sizes) for _ in range(m)]).cuda()
    names["slot_of"] = torch.tensor([i for m in sizes for i in range(m)]).cuda()
    names["row_of"] = torch.tensor(row_of).cuda()
    exec(example("kept_lse"), names)
    torch.cuda.synchronize()
    q, lse, kept, G = names["q"].double(), names["lse"].double(), 0, HQ // HKV
    for b in range(B):
        slots = names["path"][b, :names["path_len"][b]].tolist()
        kept += len(slots)
        for h in range(HKV):
            k = rows64(k_cache, table[b], at[b] + len(slots), h, False)
            want = torch.zeros(names["weights"].shape[2], dtype=torch.float64, device="cuda")
            for i, slot in enumerate(slots):
                for head in range(h * G, h * G + G):
                    row = row_of[b] + slot
                    x = k[:at[b] + i + 1] @ q[row, head] * D ** -0.5 - lse[row, head]
                    want[:at[b] + i + 1] += torch.exp(x)
            # every row's weights sum to 1 (lse is within 2e-4)
            assert abs(want.sum().item() / (len(slots) * G) - 1) < 4e-4
            old = before[b, h].double()
            got = names["weights"][b, h].double()
            assert ((got - old - want).abs() <= 2.0 ** -17 * want + 2.0 ** -20 * old).all(), (b, h)
    assert kept > 3 or max(sizes) < 4
