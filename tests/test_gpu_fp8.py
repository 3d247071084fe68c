"""The 8-bit cache: written, read back and attended to, against the definitions in 64 bits."""
import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, LSE, Layout, cache8, normal, o_bound, pow2, quantise, rotate

pytestmark = pytest.mark.gpu

DECODE = [(1, [(0, 1)]), (17, [(16, 1)]), (1000, [(999, 1)]), (4097, [(4096, 1)]), (700, [(640, 1)])]
CHUNKS = [(1500, [(900, 200)]), (40, []), (2111, [(30, 5), (64, 64), (800, 130), (2000, 111)]), (333, [(0, 333)])]
PROMPT = [(1700, [(0, 1700)])]
LAYOUTS = {"decode": DECODE, "chunks": CHUNKS, "prompt": PROMPT}


def forward(lay, plan, q, cache, table=None, lse=True, ws=None):
    o = torch.full((lay.rows, lay.hq, lay.d), float("nan"), dtype=torch.bfloat16, device="cuda")
    s = torch.full((lay.rows, lay.hq), float("nan"), device="cuda") if lse else None
    if ws is None:
        ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    msa.msa_fp8_forward(plan, q, *cache[:4], lay.table if table is None else table, o, s, ws)
    torch.cuda.synchronize()
    return o, s


def check(o, lse, ref, precise=False):
    ro, rl, mag = ref
    assert torch.isfinite(o).all()
    far = (o.double() - ro).abs() / o_bound(ro, mag, precise)
    assert (far <= 1).all(), far.max()
    if lse is not None:
        assert (lse.double() - rl).abs().max() <= LSE


@pytest.mark.parametrize("heads", [(4, 4, 64), (8, 2, 128), (32, 8, 128), (64, 1, 64), (256, 1, 128), (15, 3, 64)], ids=str)
@pytest.mark.parametrize("seqs", LAYOUTS)
def test_forward(heads, seqs):
    lay = Layout(LAYOUTS[seqs], *heads, seed=1)
    cache = cache8(lay, 3)
    q = normal(4, lay.rows, lay.hq, lay.d)
    check(*forward(lay, lay.plan(msa), q, cache), lay.attend(q, cache[4], cache[5]))


@pytest.mark.parametrize("heads", [(8, 2, 128), (6, 2, 64)], ids=str)
@pytest.mark.parametrize("rows", [32, 128, 256])
@pytest.mark.parametrize("split", [0, 64, 192])
@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 70), (90, 3), (1000, 0), (1, 0)])
def test_widths_splits_precise_windows(heads, rows, split, precise, window, sinks):
    lay = Layout(CHUNKS, *heads, seed=2)
    cache = cache8(lay, 5)
    q = normal(6, lay.rows, lay.hq, lay.d)
    flags = {32: msa.MSA_PLAN_TILE_ROWS_32, 128: msa.MSA_PLAN_TILE_ROWS_128, 256: msa.MSA_PLAN_TILE_ROWS_256}[rows]
    plan = lay.plan(msa, window, sinks, flags=flags | (msa.MSA_PLAN_PRECISE_WEIGHTS if precise else 0), kv_split_tokens=split)
    check(*forward(lay, plan, q, cache), lay.attend(q, cache[4], cache[5], window, sinks), precise)


@pytest.mark.parametrize("precise", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_many_narrow_tiles(d, precise):
    """128-row tiles, more than one for each CU: the form whose waves both copy and compute.  Over both kinds of cache."""
    lay = Layout([(260 + 7 * i, [(100, 128 + i)]) for i in range(24)], 32, 8, d, seed=3)
    cache = cache8(lay, 7)
    q = normal(8, lay.rows, lay.hq, lay.d)
    k16, v16 = cache[4].to(torch.bfloat16), cache[5].to(torch.bfloat16)
    for window in (0, 140):
        plan = lay.plan(msa, window, 2, flags=msa.MSA_PLAN_TILE_ROWS_128 | (msa.MSA_PLAN_PRECISE_WEIGHTS if precise else 0))
        assert plan.info()["num_workgroups"] > 256
        ref = lay.attend(q, cache[4], cache[5], window, 2)
        check(*forward(lay, plan, q, cache), ref, precise)
        o, lse = torch.empty_like(q), torch.empty(lay.rows, 32, device="cuda")
        ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
        msa.msa_forward(plan, q, k16, v16, lay.table, o, lse, ws)
        check(o, lse, ref, precise)


def test_long_rows():
    """Past 64 half-steps a wave and 128 steps a tile, where block ids are loaded anew."""
    lay = Layout([(30000, [(29999, 1)]), (20011, [(20000, 9)])], 8, 2, 128, seed=4)
    cache = cache8(lay, 9)
    q = normal(10, lay.rows, lay.hq, lay.d)
    ref = lay.attend(q, cache[4], cache[5])
    for flags in (0, msa.MSA_PLAN_NO_AUTO_SPLIT, msa.MSA_PLAN_NO_AUTO_SPLIT | msa.MSA_PLAN_TILE_ROWS_128,
                  msa.MSA_PLAN_NO_AUTO_SPLIT | msa.MSA_PLAN_TILE_ROWS_256):
        check(*forward(lay, lay.plan(msa, flags=flags), q, cache), ref)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 4, 64)], ids=str)
@pytest.mark.parametrize("seqs", LAYOUTS)
def test_same_as_bf16_cache(heads, seqs):
    """The values are bf16 numbers: over a bf16 cache of them the attention agrees to the rounding of both sides."""
    lay = Layout(LAYOUTS[seqs], *heads, seed=5)
    cache = cache8(lay, 11)
    q = normal(12, lay.rows, lay.hq, lay.d)
    plan = lay.plan(msa, flags=msa.MSA_PLAN_PRECISE_WEIGHTS)
    o, lse = forward(lay, plan, q, cache)
    k16, v16 = cache[4].to(torch.bfloat16), cache[5].to(torch.bfloat16)
    assert torch.equal(k16.double(), cache[4]) and torch.equal(v16.double(), cache[5])
    o2, lse2 = torch.empty_like(o), torch.empty_like(lse)
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    msa.msa_forward(plan, q, k16, v16, lay.table, o2, lse2, ws)
    ref = lay.attend(q, cache[4], cache[5])
    assert ((o.double() - o2.double()).abs() <= 2 * o_bound(ref[0], ref[2], True)).all()
    assert (lse - lse2).abs().max() <= 1e-5  # scores in another order of 32-bit sums


def test_values_behind_a_row_and_stale_blocks():
    """Numbers past the rows (finite) and blocks behind the last one do not show."""
    lay = Layout(CHUNKS, 8, 2, 128, seed=6)
    cache = list(cache8(lay, 13))
    q = normal(14, lay.rows, lay.hq, lay.d)
    plan = lay.plan(msa)
    want, wl = forward(lay, plan, q, cache)
    for b, L in enumerate(lay.lens):
        last = max(lay.pos_of[b] + [-1])
        for j in range(last + 1, -(-L // BS) * BS):
            blk = int(lay.table[b, j // BS])
            cache[0][blk, :, j % BS], cache[1][blk, :, :, j % BS] = 0x7e, 0xfe  # +-448
            cache[2][blk, :, j % BS] = cache[3][blk, :, j % BS] = 200
    got, gl = forward(lay, plan, q, cache)
    assert torch.equal(want, got) and torch.equal(wl, gl)


def test_write_read_back():
    """msa_fp8_append then msa_fp8_read: exactly the stored values, and nothing else is written."""
    for heads in ((8, 2, 128), (3, 3, 64), (8, 8, 128)):
        lay = Layout(CHUNKS, *heads, seed=7)
        cache = cache8(lay, 15)
        kn, vn = normal(16, lay.rows, lay.hkv, lay.d), normal(17, lay.rows, 2 * lay.hkv, lay.d)[:, ::2]
        msa.msa_fp8_append(lay.plan(msa), kn, vn, lay.table, *cache[:4])
        blk, at = lay.places()
        k, v = cache[4].clone(), cache[5].clone()
        k[blk, :, at], v[blk, :, :, at] = quantise(kn)[0], quantise(vn)[0]
        to = Layout(CHUNKS, *heads, seed=8, extra_blocks=9)
        for start, end, most in ((None, lay.lens, 4000), ([0, 3, 16, -7], [1500, 40, 17, 333], 4000), ([100, 0, 5, 31], [77, 0, 100, 32], 4000),
                                 (None, lay.lens, 1000), ([5, 5, 5, 5], [1 << 30, 6, 2000, -1], 1777)):
            k_out = torch.full((to.num_blocks, lay.hkv, BS, lay.d), 3.0, dtype=torch.bfloat16, device="cuda")
            v_out = torch.full((to.num_blocks, lay.hkv, lay.d, BS), 3.0, dtype=torch.bfloat16, device="cuda")
            s = None if start is None else torch.tensor(start, dtype=torch.int32, device="cuda")
            e = torch.tensor(end, dtype=torch.int32, device="cuda")
            table = lay.table.clone()
            if start and start[0] == 100:
                table[2, 3] = -1  # skipped
            msa.msa_fp8_read(lay.shape(msa), s, e, most, table, *cache[:4], to.shape(msa), to.table, k_out, v_out)
            wk, wv = torch.full_like(k_out, 3.0), torch.full_like(v_out, 3.0)
            for b, L in enumerate(lay.lens):
                # (blocks past a sequence's own have no entry in its table)
                for j in range(max(0, start[b] if start else 0), min(end[b], most, -(-L // BS) * BS)):
                    f, t = int(table[b, j // BS]), int(to.table[b, j // BS])
                    if f >= 0:
                        wk[t, :, j % BS], wv[t, :, :, j % BS] = k[f, :, j % BS].to(torch.bfloat16), v[f, :, :, j % BS].to(torch.bfloat16)
            assert torch.equal(k_out, wk) and torch.equal(v_out, wv), (heads, start)


def test_append_is_rope_append_without_rotation():
    """Frequencies of 0 turn nothing: the same bytes."""
    lay = Layout(CHUNKS, 8, 2, 128, seed=9)
    a, b = cache8(lay, 18), cache8(lay, 18)
    kn, vn = normal(19, lay.rows, 2, 128), normal(20, lay.rows, 2, 128)
    msa.msa_fp8_append(lay.plan(msa), kn, vn, lay.table, *a[:4])
    rope = msa.make_rope(torch.zeros(64, dtype=torch.float64, device="cuda"))
    msa.msa_rope_append(lay.plan(msa), rope, None, None, kn, vn, lay.table, *b[:4])
    assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))


def test_every_byte():
    """All 254 finite e4m3 numbers and many powers, through the read-back and through both attention forms
    (one key a row: o is the value)."""
    lay = Layout([(512, [(0, 512)])], 2, 2, 128, seed=10)
    codes = torch.tensor([c for c in range(256) if c & 0x7f != 0x7f], dtype=torch.uint8, device="cuda")
    i = torch.arange(lay.num_blocks * 2 * BS * 128, device="cuda")
    k = codes[i % 254].view(lay.num_blocks, 2, BS, 128)
    v = codes[(i * 7 + 3) % 254].view(lay.num_blocks, 2, 128, BS).contiguous()
    ks, vs = ((torch.arange(lay.num_blocks * 2 * BS, device="cuda") * m % 60 + 90).to(torch.uint8).view(lay.num_blocks, 2, BS) for m in (7, 11))
    kv = k.view(torch.float8_e4m3fn).double() * pow2(ks.long() - 127)[..., None]
    vv = v.view(torch.float8_e4m3fn).double() * pow2(vs.long() - 127)[:, :, None]
    k_out, v_out = torch.zeros(kv.shape, dtype=torch.bfloat16, device="cuda"), torch.zeros(vv.shape, dtype=torch.bfloat16, device="cuda")
    end = torch.tensor([512], dtype=torch.int32, device="cuda")
    msa.msa_fp8_read(lay.shape(msa), None, end, 512, lay.table, k, v, ks, vs, lay.shape(msa), lay.table, k_out, v_out)
    used = lay.table[0].long()
    assert torch.equal(k_out[used].double(), kv[used]) and torch.equal(v_out[used].double(), vv[used])
    q = torch.zeros(512, 2, 128, dtype=torch.bfloat16, device="cuda")
    want = lay.keys(0, vv, True)
    for flags in (msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256):
        o, _ = forward(lay, lay.plan(msa, 1, 0, flags=flags), q, (k, v, ks, vs))
        assert torch.equal(o.double(), want)


def test_every_channel_and_key():
    """K of one channel at a time: scores pick out that channel of q for each key."""
    for d in (64, 128):
        lay = Layout([(256, [(255, 1)]), (256, [(128, 128)])], 2, 1, d, seed=11)
        k = torch.zeros(lay.num_blocks, 1, BS, d, dtype=torch.uint8, device="cuda")
        for b in range(2):
            for j in range(256):
                k[lay.table[b, j // BS].long(), 0, j % BS, (j * 5 + b) % d] = 0x40  # 2.0
        cache = list(cache8(lay, 21))
        cache[0], cache[2] = k, torch.full_like(cache[2], 128)  # times 2
        kv = k.view(torch.float8_e4m3fn).double() * 2.0
        q = normal(22, lay.rows, 2, d)
        ref = lay.attend(q, kv, cache[5], scale=1.0)
        shape = lay.shape(msa, scale=1.0)
        for flags in (msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256):
            check(*forward(lay, lay.plan(msa, shape=shape, flags=flags), q, cache), ref)


def test_strided_and_far_caches():
    """K and V with padding between heads and blocks, offsets past 2^32 bytes."""
    lay = Layout([(600, [(500, 100)]), (333, [(332, 1)])], 4, 2, 64, seed=12)
    cache = cache8(lay, 23)
    q = normal(24, lay.rows, 4, 64)
    wants = [forward(lay, lay.plan(msa, w), q, cache) for w in (0, 90)]
    stride = (5 << 30) // lay.num_blocks // 1024 * 1024
    size = stride * lay.num_blocks
    far = [torch.zeros(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    head, tok, chan = 4096, 80, 32
    torch.as_strided(far[0], cache[0].shape, (stride, head, tok, 1)).copy_(cache[0])
    torch.as_strided(far[1], cache[1].shape, (stride, head, chan, 1)).copy_(cache[1])
    shape = lay.shape(msa, k_strides=(stride, head, tok), v_strides=(stride, head, chan))
    for w, (o, lse) in zip((0, 90), wants):
        got, gl = forward(lay, lay.plan(msa, w, shape=shape), q, far + list(cache[2:4]))
        assert torch.equal(o, got) and torch.equal(lse, gl)
    # the write and the read-back over the same strides
    kn, vn = normal(25, lay.rows, 2, 64), normal(26, lay.rows, 2, 64)
    msa.msa_fp8_append(lay.plan(msa, shape=shape), kn, vn, lay.table, far[0], far[1], cache[2], cache[3])
    msa.msa_fp8_append(lay.plan(msa), kn, vn, lay.table, *cache[:4])
    assert torch.equal(torch.as_strided(far[0], cache[0].shape, (stride, head, tok, 1)), cache[0])
    assert torch.equal(torch.as_strided(far[1], cache[1].shape, (stride, head, chan, 1)), cache[1])
    end = torch.tensor(lay.lens, dtype=torch.int32, device="cuda")
    outs = [[torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((lay.num_blocks, 2, BS, 64), (lay.num_blocks, 2, 64, BS))] for _ in range(2)]
    msa.msa_fp8_read(shape, None, end, 600, lay.table, *far, *cache[2:4], lay.shape(msa), lay.table, *outs[0])
    msa.msa_fp8_read(lay.shape(msa), None, end, 600, lay.table, *cache[:4], lay.shape(msa), lay.table, *outs[1])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_refusals():
    lay = Layout(CHUNKS, 8, 2, 128, seed=13)
    cache = cache8(lay, 27)
    q = normal(28, lay.rows, 8, 128)
    o = torch.empty_like(q)
    plan = lay.plan(msa)
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")

    def refused(text, status=msa.MSA_ERR_INVALID_ARG, p=plan, **kw):
        a = dict(q=q, k_cache=cache[0], v_cache=cache[1], k_scale=cache[2], v_scale=cache[3], block_table=lay.table, o=o, workspace=ws)
        a.update(kw)
        with pytest.raises(msa.MsaError, match=text) as e:
            msa.msa_fp8_forward(p, **a)
        assert e.value.status == status
    refused("k_cache has type", k_cache=cache[0].view(torch.bfloat16))
    refused("v_scale has", v_scale=cache[3][1:])
    refused("k_scale has type", k_scale=cache[2].to(torch.int32))
    refused("must be non-null", k_scale=None)
    refused("q has type", q=q.float())
    refused("lse has", lse=torch.zeros(3, device="cuda"))
    tree = msa.msa_plan_tree(lay.shape(msa), lay.lens, lay.indptr, lay.start, lay.length)
    refused("msa_plan_tree", msa.MSA_ERR_UNSUPPORTED, p=tree)
    odd = lay.plan(msa, shape=lay.shape(msa, k_strides=(4104, 2048, 128)))
    refused("multiples of 16", p=odd)
    for field, stride in (("k_stride_tok", 286331200), ("v_stride_dim", 33818656)):  # 15 and 127 of them: past 2^32
        wide = lay.shape(msa)
        setattr(wide, field, stride)
        refused("4 GiB", msa.MSA_ERR_UNSUPPORTED, p=lay.plan(msa, shape=wide))
    with pytest.raises(msa.MsaError, match="multiples of 16"):
        msa.msa_fp8_append(odd, normal(1, lay.rows, 2, 128), normal(2, lay.rows, 2, 128), lay.table, *cache[:4])


@pytest.mark.parametrize("window", [0, 200])
def test_a_layer(window):
    """A step as a model runs it: rotation and write, attention, then the cache back in bf16 and the next token; captured
    once and replayed with other inputs, each replay against eager calls."""
    lay = Layout([(400 + 37 * i, [(300, 100 + 37 * i - 1)] if i % 2 else [(399 + 37 * i, 1)]) for i in range(6)], 8, 2, 128, seed=14)
    plan, shape = lay.plan(msa, window, 4), lay.shape(msa)
    freq = torch.from_numpy(msa.msa_rope_freqs(128, 500000.0)[0]).cuda()
    rope = msa.make_rope(freq)
    qkv = normal(30, lay.rows, 12, 128)
    ws = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    end = torch.tensor(lay.lens, dtype=torch.int32, device="cuda")

    def buffers():
        c = cache8(lay, 29)
        return (list(c[:4]), torch.zeros(lay.rows, 8, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(lay.rows, 8, 128, dtype=torch.bfloat16, device="cuda"),
                torch.zeros(lay.rows, 8, device="cuda"), torch.zeros(lay.num_blocks, 2, BS, 128, dtype=torch.bfloat16, device="cuda"),
                torch.zeros(lay.num_blocks, 2, 128, BS, dtype=torch.bfloat16, device="cuda"))

    def step(cache, q, o, lse, k16, v16):
        msa.msa_rope_append(plan, rope, qkv[:, :8], q, qkv[:, 8:10], qkv[:, 10:], lay.table, *cache)
        msa.msa_fp8_forward(plan, q, *cache, lay.table, o, lse, ws)
        msa.msa_fp8_read(shape, None, end, 700, lay.table, *cache, shape, lay.table, k16, v16)
    a, b = buffers(), buffers()
    step(*a)
    torch.cuda.synchronize()
    cache, q, o, lse, k16, v16 = a
    kv = cache[0].view(torch.float8_e4m3fn).double() * pow2(cache[2].long() - 127)[..., None]
    vv = cache[1].view(torch.float8_e4m3fn).double() * pow2(cache[3].long() - 127)[:, :, None]
    check(o, lse, lay.attend(q, kv, vv, window, 4))
    want = rotate(qkv[:, :8], lay.pos, freq, 0)
    assert ((q.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()
    # the bf16 cache goes on where the 8-bit one was: the same attention to the rounding of both
    o2 = torch.zeros_like(o)
    msa.msa_forward(plan, q, k16, v16, lay.table, o2, None, ws)
    ref = lay.attend(q, kv, vv, window, 4)
    assert ((o.double() - o2.double()).abs() <= 2 * o_bound(ref[0], ref[2])).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(*b)
    for seed in (31, 32, 33):
        qkv.copy_(normal(seed, *qkv.shape))
        graph.replay()
        torch.cuda.synchronize()
        step(*a)
        torch.cuda.synchronize()
        flat = lambda t: [*t[0], *t[1:]]  # noqa: E731
        assert all(torch.equal(x, y) for x, y in zip(flat(a), flat(b)))


def test_two_graphs_and_streams():
    """Two captured calls with workspaces of their own, replayed side by side on two streams."""
    lay = Layout([(9000, [(8999, 1)]), (5000, [(4990, 10)])], 8, 2, 128, seed=15)
    cache, plan = cache8(lay, 33), lay.plan(msa)
    need = plan.info()["workspace_bytes"]
    assert need > 0
    qs = [normal(s, lay.rows, 8, 128) for s in (1, 2)]
    want = [forward(lay, plan, q, cache)[0] for q in qs]
    outs, graphs = [torch.zeros_like(q) for q in qs], []
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in qs]
    for q, o, ws in zip(qs, outs, spaces):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            msa.msa_fp8_forward(plan, q, *cache[:4], lay.table, o, None, ws)
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in qs]
    for _ in range(4):
        for o in outs:
            o.zero_()
        torch.cuda.synchronize()
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs))
