"""Rows of few keys in plans of msa_plan_window: two terms a weight by the window and the sinks alone, whatever else
the batch holds."""
import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, LSE, Layout, cache8, normal, o_bound

pytestmark = pytest.mark.gpu

SHORT = (90, [(0, 90)])  # no row has a key behind a window of 100


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


def caches(lay, seed):
    c = cache8(lay, seed)
    return {"bf16": (c[4].to(torch.bfloat16), c[5].to(torch.bfloat16)), "fp8": c[:4]}, c[4], c[5]


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("window,sinks,precise", [(100, 4, True), (128, 0, True), (90, 38, True), (100, 29, False), (129, 0, False),
                                                  (90, 9000, False)])
def test_a_window_that_hides_nothing(window, sinks, precise, cache):
    """The causal plan, with MSA_PLAN_PRECISE_WEIGHTS for up to 128 keys: the same bits."""
    lay = Layout([SHORT], 8, 2, 128, seed=1)
    both, _, _ = caches(lay, 2)
    q = normal(3, lay.rows, 8, 128)
    got = run(lay, lay.plan(msa, window, sinks), q, both[cache])
    one = run(lay, lay.plan(msa), q, both[cache])
    two = run(lay, lay.plan(msa, flags=msa.MSA_PLAN_PRECISE_WEIGHTS), q, both[cache])
    assert not torch.equal(one[0], two[0])
    assert all(torch.equal(a, b) for a, b in zip(got, two if precise else one))


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("seqs", [[SHORT], [SHORT, (5000, [(4900, 100)])], [(3000, [(2999, 1)]), SHORT]], ids=["alone", "chunk", "token"])
def test_weights_do_not_depend_on_the_batch(seqs, cache):
    """Few keys of much weight, in steps before the rows' own: the bound of two terms, alone and next to longer rows."""
    lay = Layout(seqs, 8, 2, 64, seed=4)
    both, k, v = caches(lay, 5)
    q = normal(6, lay.rows, 8, 64) * 3
    o, lse = run(lay, lay.plan(msa, 100, 4), q, both[cache])
    ro, rl, mag = lay.attend(q, k, v, 100, 4)
    assert ((o.double() - ro).abs() <= o_bound(ro, mag, True)).all()
    assert (lse.double() - rl).abs().max() <= LSE
