"""Items of up to 32 rows whose K and V come by way of LDS (windows, 8-bit caches): the copies' places for
any strides, rows of many half-steps, and stages that one item leaves to the next."""
import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, LSE, Layout, cache8, normal, o_bound

pytestmark = pytest.mark.gpu


def run(lay, plan, q, cache):
    o = torch.full((lay.rows, lay.hq, lay.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((lay.rows, lay.hq), float("nan"), device="cuda")
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    if len(cache) == 4:
        msa.msa_fp8_forward(plan, q, *cache, lay.table, o, lse, ws)
    else:
        msa.msa_forward(plan, q, *cache, lay.table, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def check(got, ref):
    (o, lse), (ro, rl, mag) = got, ref
    assert ((o.double() - ro).abs() <= o_bound(ro, mag)).all()
    assert (lse.double() - rl).abs().max() <= LSE


def caches(lay, seed):
    """((bf16 K, V), (8-bit K, V, powers), their values): both hold the same numbers."""
    c = cache8(lay, seed)
    return (c[4].to(torch.bfloat16), c[5].to(torch.bfloat16)), c[:4], c[4], c[5]


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("window,sinks", [(9001, 100), (12345, 0), (0, 0)])
def test_rows_of_many_half_steps(heads, window, sinks):
    """Uncut: up to 98 half-steps a wave, where the ids of the first 64 are held and later ones looked up."""
    lay = Layout([(12500, [(12499, 1)]), (9007, [(9000, 3)]), (70, [(69, 1)])], *heads, seed=1)
    bf16, fp8, k, v = caches(lay, 2)
    q = normal(3, lay.rows, lay.hq, lay.d)
    ref = lay.attend(q, k, v, window, sinks)
    plan = lay.plan(msa, window, sinks, flags=msa.MSA_PLAN_NO_AUTO_SPLIT)
    assert plan.info()["max_splits"] == 1 and plan.info()["tile_rows"] == 32
    for cache in (bf16, fp8):
        check(run(lay, plan, q, cache), ref)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("window,sinks", [(150, 20), (0, 0)])
def test_strides(heads, window, sinks):
    """Tokens, channels, heads and blocks apart from each other, in memory that is otherwise NaN."""
    lay = Layout([(1, [(0, 1)]), (333, [(332, 1)]), (600, [(590, 7)])], *heads, seed=4)
    d, bf16_cache = lay.d, window > 0
    bf16, fp8, k, v = caches(lay, 5)
    # elements: a token of K, a channel of V (multiples of 16), a head and a block, with room between them
    tok, chan = d + 16, 32
    k_head, v_head = BS * tok + 48, d * chan + 16
    k_block, v_block = lay.hkv * k_head + 80, lay.hkv * v_head + 32
    plan = lay.plan(msa, window, sinks, shape=lay.shape(msa, k_strides=(k_block, k_head, tok), v_strides=(v_block, v_head, chan)))
    q = normal(6, lay.rows, lay.hq, d)
    ref = lay.attend(q, k, v, window, sinks)

    def spread(x, size, strides, bad):
        base = torch.full((lay.num_blocks * size,), bad, dtype=x.dtype, device="cuda")
        base.as_strided(x.shape, strides).copy_(x)
        return base
    for cache, bad in ((bf16, float("nan")), (fp8, 0x7f)):
        kc = spread(cache[0], k_block, (k_block, k_head, tok, 1), bad)
        vc = spread(cache[1], v_block, (v_block, v_head, chan, 1), bad)
        if bf16_cache or len(cache) == 4:
            check(run(lay, plan, q, (kc, vc, *cache[2:])), ref)


@pytest.mark.parametrize("heads", [(32, 8, 128), (16, 16, 64)], ids=str)
@pytest.mark.parametrize("window,sinks", [(100, 3), (0, 0)])
def test_many_items_a_workgroup(heads, window, sinks):
    """Several items a workgroup, of one half-step to many: each wave's stage is where the item before left its partial
    output.  The rows' bits are those of the same rows in plans of few items."""
    lens = [1, 40, 17, 300, 33, 129, 64, 16] * 25
    lay = Layout([(n, [(n - 1, 1)]) for n in lens], *heads, seed=7)
    bf16, fp8, k, v = caches(lay, 8)
    q = normal(9, lay.rows, lay.hq, lay.d)
    ref = lay.attend(q, k, v, window, sinks)
    plan = lay.plan(msa, window, sinks, flags=msa.MSA_PLAN_NO_AUTO_SPLIT)
    i = plan.info()
    assert i["tile_rows"] == 32 and i["num_work"] >= 3 * i["num_workgroups"] / 2
    for cache in (bf16, fp8):
        got = run(lay, plan, q, cache)
        check(got, ref)
        for _ in range(3):
            again = run(lay, plan, q, cache)
            assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
        few = Layout([(n, [(n - 1, 1)]) for n in lens[:8]], *heads, seed=7)
        few.table = lay.table[:8, :few.max_blocks].contiguous()
        few.num_blocks = lay.num_blocks
        o, lse = run(few, few.plan(msa, window, sinks, flags=msa.MSA_PLAN_NO_AUTO_SPLIT), q[:8].contiguous(), cache)
        assert torch.equal(o, got[0][:8]) and torch.equal(lse, got[1][:8])
