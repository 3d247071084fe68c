"""Windowed attention with sinks (msa_plan_window) against the definition in 64 bits."""

import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, LSE, Layout, normal, o_bound

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (8, 2, 128), (32, 8, 128), (64, 1, 64), (256, 1, 128)]


def call(lay, plan, q, k, v, table=None, lse=True):
    o = torch.full((lay.rows, lay.hq, lay.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    s = torch.full((lay.rows, lay.hq), float("nan"), device="cuda") if lse else None
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    msa.msa_forward(plan, q, k, v, lay.table if table is None else table, o, s, ws)
    torch.cuda.synchronize()
    return o, s


def check(lay, o, lse, ref, precise=False):
    ro, rl, mag = ref
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    assert ((o.double() - ro).abs() <= o_bound(ro, mag, precise)).all(), ((o.double() - ro).abs() / o_bound(ro, mag, precise)).max()
    assert (lse.double() - rl).abs().max() <= LSE


def inputs(lay, seed):
    return (normal(seed, lay.rows, lay.hq, lay.d), normal(seed + 1, lay.num_blocks, lay.hkv, BS, lay.d),
            normal(seed + 2, lay.num_blocks, lay.hkv, lay.d, BS))


DECODE = [(1, [(0, 1)]), (17, [(16, 1)]), (1000, [(999, 1)]), (4097, [(4096, 1)]), (700, [(640, 1)])]
CHUNKS = [(1500, [(900, 200)]), (40, []), (2111, [(30, 5), (64, 64), (800, 130), (2000, 111)]), (333, [(0, 333)])]
PROMPT = [(1700, [(0, 1700)])]


@pytest.mark.parametrize("heads", HEADS[:3], ids=str)
@pytest.mark.parametrize("seqs", [DECODE, CHUNKS, PROMPT], ids=["decode", "chunks", "prompt"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (16, 0), (63, 4), (64, 64), (65, 1), (100, 65), (500, 4), (777, 200),
                                          (5000, 0), (300, 5000)])
def test_definition(seqs, heads, window, sinks):
    lay = Layout(seqs, *heads, seed=window)
    q, k, v = inputs(lay, 10 + window)
    plan = lay.plan(msa, window, sinks)
    o, lse = call(lay, plan, q, k, v)
    check(lay, o, lse, lay.attend(q, k, v, window, sinks))


@pytest.mark.parametrize("rows", [32, 128, 256])
@pytest.mark.parametrize("split", [0, 64, 192])
@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64)], ids=str)
def test_widths_splits_precise(rows, split, precise, heads):
    lay = Layout(CHUNKS, *heads, seed=4)
    q, k, v = inputs(lay, 60)
    flags = {32: msa.MSA_PLAN_TILE_ROWS_32, 128: msa.MSA_PLAN_TILE_ROWS_128, 256: msa.MSA_PLAN_TILE_ROWS_256}[rows]
    flags |= msa.MSA_PLAN_PRECISE_WEIGHTS if precise else 0
    for window, sinks in ((300, 70), (90, 3), (1000, 0)):
        plan = lay.plan(msa, window, sinks, flags=flags, kv_split_tokens=split)
        o, lse = call(lay, plan, q, k, v)
        check(lay, o, lse, lay.attend(q, k, v, window, sinks), precise)


@pytest.mark.parametrize("heads", HEADS[3:], ids=str)
def test_wide_groups(heads):
    lay = Layout([(300, [(250, 50)]), (900, [(899, 1)])], *heads, seed=5)
    q, k, v = inputs(lay, 70)
    o, lse = call(lay, lay.plan(msa, 70, 2), q, k, v)
    check(lay, o, lse, lay.attend(q, k, v, 70, 2))


@pytest.mark.parametrize("window,sinks", [(1, 0), (2, 1), (5, 64), (64, 0), (65, 4), (128, 17), (1000, 1), (333, 129)])
@pytest.mark.parametrize("seqs", [DECODE, CHUNKS, PROMPT], ids=["decode", "chunks", "prompt"])
def test_every_key_counts_once(seqs, window, sinks):
    """With q = 0 every visible key weighs the same: lse is the logarithm of their number, o their mean."""
    lay = Layout(seqs, 4, 2, 64, seed=window)
    q, k, v = inputs(lay, 80)
    o, lse = call(lay, lay.plan(msa, window, sinks), torch.zeros_like(q), k, v)
    p = lay.pos.double()
    count = torch.where(p < window, p + 1, window + torch.clamp(p - window + 1, max=sinks))
    # (a key more or less moves it by 1 / 1133 at least; sums of up to 1133 equal numbers in 32 bits by 2e-6)
    assert (lse.double() - count.log()[:, None]).abs().max() <= 1e-5
    check(lay, o, lse, lay.attend(torch.zeros_like(q), k, v, window, sinks))


def test_window_past_the_context_is_causal():
    """The same bits as msa_plan's."""
    lay = Layout(CHUNKS, 8, 2, 128, seed=6)
    q, k, v = inputs(lay, 90)
    a, la = call(lay, lay.plan(msa), q, k, v)
    for window, sinks in ((2111, 0), (1 << 30, 7), ((1 << 31) - 1, (1 << 31) - 1)):
        b, lb = call(lay, lay.plan(msa, window, sinks), q, k, v)
        assert torch.equal(a, b) and torch.equal(la, lb)


@pytest.mark.parametrize("seqs", [DECODE, CHUNKS], ids=["decode", "chunks"])
@pytest.mark.parametrize("window,sinks", [(40, 5), (200, 0), (128, 64)])
def test_blocks_out_of_the_window_are_not_read(seqs, window, sinks):
    """Entries of blocks that no row can see may name any block: here ones of NaN and, in the table that the check
    takes, none."""
    lay = Layout(seqs, 8, 2, 128, seed=7)
    q, k, v = inputs(lay, 100)
    plan = lay.plan(msa, window, sinks)
    want, wl = call(lay, plan, q, k, v)
    table = lay.table.clone()
    bad = lay.num_blocks  # a block of NaN behind the others
    k2 = torch.cat((k, torch.full_like(k[:1], float("nan"))))
    v2 = torch.cat((v, torch.full_like(v[:1], float("nan"))))
    hidden = 0
    for b, pos in enumerate(lay.pos_of):
        used = set()
        if pos:
            used |= set(range(max(0, pos[0] - window + 1) // BS, pos[-1] // BS + 1)) | set(range(-(-min(sinks, pos[-1] + 1) // BS)))
        for i in range(lay.max_blocks):
            if i not in used:
                table[b, i] = bad
                hidden += 1
    assert hidden > 5
    got, gl = call(lay, plan, q, k2, v2, table)
    assert torch.equal(want, got) and torch.equal(wl, gl)
    host = table.cpu().numpy().copy()
    host[host == bad] = -1
    msa.msa_check_block_table(plan, host)
    msa.msa_check_block_table(plan, torch.where(table == bad, -1, table))


def test_nan_before_the_window_stays_out():
    """K and V of hidden positions of the window's own first block: K may be NaN, weights and sums do not see it."""
    lay = Layout([(200, [(150, 50)])], 8, 2, 128, seed=8)
    q, k, v = inputs(lay, 110)
    plan = lay.plan(msa, 60, 3)
    want, wl = call(lay, plan, q, k, v)
    for j in (3, 5, 15, 85, 90):  # 85, 90: before the first row's window (91), in blocks that are read
        k[lay.table[0, j // BS].long(), :, j % BS] = float("nan")
    got, gl = call(lay, plan, q, k, v)
    assert torch.equal(want, got) and torch.equal(wl, gl)


def test_rows_do_not_depend_on_their_tile():
    """A row has the same bits alone, in a chunk and in tiles of any width, where nothing is split."""
    lay = Layout([(1200, [(700, 300)])], 8, 2, 128, seed=9)
    q, k, v = inputs(lay, 120)
    base = None
    for flags in (msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256):
        o, lse = call(lay, lay.plan(msa, 250, 4, flags=flags | msa.MSA_PLAN_NO_AUTO_SPLIT), q, k, v)
        if base is not None:
            assert torch.equal(o, base[0]) and torch.equal(lse, base[1])
        base = (o, lse)


def test_noalloc_stream_graph():
    """msa_forward_noalloc, another stream, and a graph replayed with changed inputs."""
    lay = Layout(CHUNKS, 8, 2, 128, seed=10)
    q, k, v = inputs(lay, 130)
    plan = lay.plan(msa, 150, 4)
    want, wl = call(lay, plan, q, k, v)
    o, lse = torch.zeros_like(want), torch.zeros_like(wl)
    msa.msa_forward_noalloc(plan, q, k, v, lay.table, o, lse)
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(lse, wl)
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o.zero_()
    with torch.cuda.stream(side):
        msa.msa_forward(plan, q, k, v, lay.table, o, lse, ws)
    side.synchronize()
    assert torch.equal(o, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        msa.msa_forward(plan, q, k, v, lay.table, o, lse, ws)
    for seed in (1, 2, 3):
        q.copy_(normal(seed, *q.shape))
        graph.replay()
        torch.cuda.synchronize()
        again, al = call(lay, plan, q, k, v)
        assert torch.equal(o, again) and torch.equal(lse, al)


def test_far_blocks():
    """Cache offsets past 2^31 elements."""
    lay = Layout([(600, [(500, 100)])], 4, 1, 64, seed=11)
    q, k, v = inputs(lay, 140)
    plan = lay.plan(msa, 100, 2)
    want, wl = call(lay, plan, q, k, v)
    stride = (1 << 31) // lay.num_blocks // 1024 * 1024 * 2
    size = stride * (lay.num_blocks - 1) + BS * lay.d
    far_k, far_v = (torch.zeros(size, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    torch.as_strided(far_k, k.shape, (stride, BS * lay.d, lay.d, 1)).copy_(k)
    torch.as_strided(far_v, v.shape, (stride, BS * lay.d, BS, 1)).copy_(v)
    shape = lay.shape(msa, k_strides=(stride, BS * lay.d, lay.d), v_strides=(stride, BS * lay.d, BS))
    assert (lay.num_blocks - 1) * stride > 1 << 31
    o, lse = call(lay, lay.plan(msa, 100, 2, shape=shape), q, far_k, far_v)
    assert torch.equal(o, want) and torch.equal(lse, wl)


def test_append_takes_the_plan():
    lay = Layout(CHUNKS, 8, 2, 128, seed=12)
    _, k, v = inputs(lay, 150)
    kn, vn = normal(1, lay.rows, 2, 128), normal(2, lay.rows, 2, 128)
    k1, v1 = k.clone(), v.clone()
    msa.msa_kv_append(lay.plan(msa), kn, vn, lay.table, k, v)
    msa.msa_kv_append(lay.plan(msa, 33, 4), kn, vn, lay.table, k1, v1)
    assert torch.equal(k, k1) and torch.equal(v, v1)


def test_key_weights_refuse_the_plan():
    lay = Layout(CHUNKS, 8, 2, 128, seed=13)
    q, k, v = inputs(lay, 160)
    w = torch.zeros(len(lay.seqs), 2, lay.max_blocks * BS, device="cuda")
    with pytest.raises(msa.MsaError, match="msa_plan_window") as e:
        msa.msa_kv_weights(lay.plan(msa, 9), q, k, lay.table, torch.zeros(lay.rows, 8, device="cuda"), w)
    assert e.value.status == msa.MSA_ERR_UNSUPPORTED
