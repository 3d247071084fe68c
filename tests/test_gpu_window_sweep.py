"""A seeded sweep of windowed and 8-bit attention: random layouts, heads, windows, sinks, tile widths, forced splits
and precise weights, each compared in full with the definition in 64 bits."""
import random

import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, LSE, Layout, cache8, normal, o_bound

pytestmark = pytest.mark.gpu


def case(seed):
    r = random.Random(seed)
    heads = r.choice(((4, 4, 64), (8, 2, 128), (32, 8, 128), (12, 4, 64), (7, 7, 128), (20, 1, 64), (40, 2, 128)))
    seqs = []
    for _ in range(r.randint(1, 5)):
        at, segs = r.choice((0, 0, 5, 100, 1000, 3000)), []
        for _ in range(r.randint(0, 3)):
            n = r.choice((1, 1, 3, 15, 16, 17, 63, 64, 65, 130, 300))
            segs.append((at, n))
            at += n + r.choice((0, 1, 30, 200, 900))
        seqs.append((at + r.randint(0, 20) if at else 1, segs))
    if not any(segs for _, segs in seqs):
        seqs.append((100, [(99, 1)]))
    window = r.choice((0, 1, 7, 16, 50, 64, 100, 200, 640, 1500))
    sinks = r.choice((0, 0, 1, 4, 16, 63, 64, 70, 300)) if window else 0
    fp8 = window == 0 or r.random() < 0.5
    flags = r.choice((0, 0, msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256,
                      msa.MSA_PLAN_TILE_ROWS_32 if heads[0] // heads[1] <= 32 else 0))
    precise = r.random() < 0.25
    kw = dict(flags=flags | (msa.MSA_PLAN_PRECISE_WEIGHTS if precise else 0) | r.choice((0, 0, msa.MSA_PLAN_NO_AUTO_SPLIT)),
              kv_split_tokens=r.choice((0, 0, 0, 64, 128, 320)))
    return heads, seqs, window, sinks, fp8, precise, kw


@pytest.mark.parametrize("seed", range(160))
def test_sweep(seed):
    heads, seqs, window, sinks, fp8, precise, kw = case(seed)
    lay = Layout(seqs, *heads, seed=seed)
    plan = lay.plan(msa, window, sinks, **kw)
    q = normal(seed, lay.rows, lay.hq, lay.d)
    o = torch.full((lay.rows, lay.hq, lay.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((lay.rows, lay.hq), float("nan"), device="cuda")
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    if fp8:
        cache = cache8(lay, seed)
        k, v = cache[4], cache[5]
        msa.msa_fp8_forward(plan, q, *cache[:4], lay.table, o, lse, ws)
    else:
        k, v = normal(seed + 1, lay.num_blocks, lay.hkv, BS, lay.d), normal(seed + 2, lay.num_blocks, lay.hkv, lay.d, BS)
        msa.msa_forward(plan, q, k, v, lay.table, o, lse, ws)
    torch.cuda.synchronize()
    ro, rl, mag = lay.attend(q, k, v, window, sinks)
    # (two terms a weight with the flag, and where a window hides keys and leaves up to 128; one that hides nothing is
    # msa_plan's, whose weights are bf16 numbers off their row's own step)
    hides = 0 < window < int(lay.pos.max()) + 1
    far = (o.double() - ro).abs() / o_bound(ro, mag, precise or (hides and window + sinks <= 128))
    assert torch.isfinite(o).all() and (far <= 1).all(), far.max()
    assert (lse.double() - rl).abs().max() <= LSE
