"""Windows over the 8-bit cache where a wrong block, scale or key would hide among many right ones: blocks that are
not to be read, hidden keys, and counts of equal weights, in tiles of every width."""
import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, Layout, cache8, normal, o_bound

pytestmark = pytest.mark.gpu

DECODE = [(1, [(0, 1)]), (17, [(16, 1)]), (1000, [(999, 1)]), (4097, [(4096, 1)]), (700, [(640, 1)])]
CHUNKS = [(1500, [(900, 200)]), (40, []), (2111, [(30, 5), (64, 64), (800, 130), (2000, 111)]), (333, [(0, 333)])]
LAYOUTS = {"decode": DECODE, "chunks": CHUNKS, "prompt": [(1700, [(0, 1700)])]}
WIDTHS = {32: msa.MSA_PLAN_TILE_ROWS_32, 128: msa.MSA_PLAN_TILE_ROWS_128, 256: msa.MSA_PLAN_TILE_ROWS_256}
NAN, HUGE = 0x7f, 255  # of e4m3; a power that makes every number infinite


def forward(lay, plan, q, cache, table=None):
    o = torch.full((lay.rows, lay.hq, lay.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((lay.rows, lay.hq), float("nan"), device="cuda")
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    msa.msa_fp8_forward(plan, q, *cache, lay.table if table is None else table, o, lse, ws)
    torch.cuda.synchronize()
    return o, lse


def equal(a, b):
    return torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("rows", WIDTHS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs", ["decode", "chunks"])
@pytest.mark.parametrize("window,sinks", [(40, 5), (200, 0), (128, 64)])
def test_blocks_out_of_the_window_are_not_read(seqs, window, sinks, d, rows):
    """Entries of blocks before the first row's window and behind the sinks name one whose numbers are NaN and whose
    powers make any number infinite."""
    lay = Layout(LAYOUTS[seqs], 8, 2, d, seed=7)
    cache = cache8(lay, 8)[:4]
    q = normal(9, lay.rows, 8, d)
    want = forward(lay, lay.plan(msa, window, sinks, flags=WIDTHS[rows]), q, cache)
    assert torch.isfinite(want[0]).all() and torch.isfinite(want[1]).all()
    bad, table, hidden = lay.num_blocks, lay.table.clone(), 0
    cache = [torch.cat((x, torch.full_like(x[:1], y))) for x, y in zip(cache, (NAN, NAN, HUGE, HUGE))]
    for b, pos in enumerate(lay.pos_of):
        used = set()
        if pos:
            used |= set(range(max(0, pos[0] - window + 1) // BS, pos[-1] // BS + 1)) | set(range(-(-min(sinks, pos[-1] + 1) // BS)))
        for i in set(range(lay.max_blocks)) - used:
            table[b, i] = bad
            hidden += 1
    assert hidden > 5
    shape = lay.shape(msa)
    shape.num_blocks += 1
    plan = lay.plan(msa, window, sinks, shape=shape, flags=WIDTHS[rows])
    assert equal(want, forward(lay, plan, q, cache, table))


@pytest.mark.parametrize("rows", WIDTHS)
@pytest.mark.parametrize("d", [64, 128])
def test_nan_before_the_window_stays_out(d, rows):
    """K of hidden positions in blocks that are read may be NaN, and infinite by its power."""
    lay = Layout([(200, [(150, 50)])], 8, 2, d, seed=8)
    cache = cache8(lay, 10)[:4]
    q = normal(11, lay.rows, 8, d)
    plan = lay.plan(msa, 60, 3, flags=WIDTHS[rows])
    want = forward(lay, plan, q, cache)
    for j in (3, 5, 15, 85, 90):  # 85, 90: before the first row's window (91)
        blk = lay.table[0, j // BS].long()
        cache[0][blk, :, j % BS], cache[2][blk, :, j % BS] = NAN, HUGE
    assert torch.isfinite(want[0]).all() and equal(want, forward(lay, plan, q, cache))


@pytest.mark.parametrize("rows", WIDTHS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (5, 64), (64, 0), (65, 4), (128, 17), (1000, 1), (333, 129)])
@pytest.mark.parametrize("seqs", LAYOUTS)
def test_every_key_counts_once(seqs, window, sinks, rows):
    """With q = 0 every visible key weighs the same: lse is the logarithm of their number, o their mean."""
    lay = Layout(LAYOUTS[seqs], 4, 2, 64, seed=window)
    cache = cache8(lay, 12)
    q = torch.zeros(lay.rows, 4, 64, dtype=torch.bfloat16, device="cuda")
    o, lse = forward(lay, lay.plan(msa, window, sinks, flags=WIDTHS[rows]), q, cache[:4])
    p = lay.pos.double()
    count = torch.where(p < window, p + 1, window + torch.clamp(p - window + 1, max=sinks))
    # (a key more or less moves it by 1 / 1133 at least; sums of up to 1133 equal numbers in 32 bits by 2e-6)
    assert (lse.double() - count.log()[:, None]).abs().max() <= 1e-5
    ro, _, mag = lay.attend(q, cache[4], cache[5], window, sinks)
    assert ((o.double() - ro).abs() <= o_bound(ro, mag)).all()


@pytest.mark.parametrize("cache", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_rows_do_not_depend_on_their_tile(d, cache):
    """A row has the same bits in a tile of its own, in a chunk and in tiles of 128 and 256 rows, where nothing is
    split."""
    lay = Layout([(1200, [(700, 300)])], 8, 2, d, seed=9)
    both, q = cache8(lay, 13), normal(14, lay.rows, 8, d)
    k16, v16 = both[4].to(torch.bfloat16), both[5].to(torch.bfloat16)

    def run(seqs, q, flags):
        one = Layout(seqs, 8, 2, d, seed=9)  # (the same blocks: they go by the lengths and the seed)
        assert torch.equal(one.table, lay.table)
        plan = one.plan(msa, 250, 4, flags=flags | msa.MSA_PLAN_NO_AUTO_SPLIT)
        if cache == "fp8":
            return forward(one, plan, q, both[:4])
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        msa.msa_forward(plan, q, k16, v16, one.table, o, lse, None)
        torch.cuda.synchronize()
        return o, lse

    for flags in (WIDTHS[128], WIDTHS[256]):
        o, lse = run(lay.seqs, q, flags)
        if flags == WIDTHS[128]:
            want = o, lse
        assert equal(want, (o, lse))
        for i in (0, 1, 63, 64, 150, 299):
            a, b = run([(1200, [(700 + i, 1)])], q[i:i + 1].contiguous(), flags)
            assert torch.equal(a[0], o[i]) and torch.equal(b[0], lse[i]), i
