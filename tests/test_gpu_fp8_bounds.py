"""The largest numbers that an 8-bit cache may be given, written, read back and attended to."""
import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, Layout, quantise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_largest_numbers(d):
    """Rows up to 247 * 2^120 are stored as 240 * 2^120 at most: finite bf16 numbers when they are read back, and in
    the sums of attention (one key a row: the output is the value)."""
    lay = Layout([(48, [(0, 48)])], 1, 1, d, seed=1)
    top = 247.0 * 2.0 ** 120
    x = torch.zeros(48, 1, d, dtype=torch.bfloat16, device="cuda")
    for i in range(48):
        x[i, 0, i] = top if i % 2 else -top
        x[i, 0, (i + 1) % d] = (225 + i % 22) * 2.0 ** 120
    assert torch.isfinite(x).all()
    want, powers = quantise(x)
    k = torch.zeros(lay.num_blocks, 1, BS, d, dtype=torch.uint8, device="cuda")
    v = torch.zeros(lay.num_blocks, 1, d, BS, dtype=torch.uint8, device="cuda")
    ks, vs = (torch.full((lay.num_blocks, 1, BS), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    msa.msa_fp8_append(lay.plan(msa), x, x, lay.table, k, v, ks, vs)
    k16 = torch.zeros(lay.num_blocks, 1, BS, d, dtype=torch.bfloat16, device="cuda")
    v16 = torch.zeros(lay.num_blocks, 1, d, BS, dtype=torch.bfloat16, device="cuda")
    end = torch.tensor([48], dtype=torch.int32, device="cuda")
    shape = lay.shape(msa)
    msa.msa_fp8_read(shape, None, end, 48, lay.table, k, v, ks, vs, shape, lay.table, k16, v16)
    blk, at = lay.places()
    assert int(powers.max()) == 247 and float(want.abs().max()) == 240.0 * 2.0 ** 120
    assert torch.equal(k16[blk, :, at].double(), want) and torch.equal(v16[blk, :, :, at].double(), want)
    q = torch.zeros(48, 1, d, dtype=torch.bfloat16, device="cuda")
    for flags in (msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256):
        o, plan = torch.empty_like(q), lay.plan(msa, 1, 0, flags=flags)
        ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
        msa.msa_fp8_forward(plan, q, k, v, ks, vs, lay.table, o, None, ws)
        assert torch.equal(o.double(), want)
