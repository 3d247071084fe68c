"""Key weights, selection and compaction of the paged cache (msa_kv_weights,
msa_kv_select, msa_kv_compact) against plain 64-bit forms (GPU only).

The weights' bar: an exponent's error in fp32 (the score's sum of D products, lse and
their difference, in units of log2: under 2^-19 for |score|, |lse| < 32) and the sums',
together 2^-17 of a key's weight, plus 2^-20 of what stood there before.
"""
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from tree_ref import attention64, paged, rows64  # noqa: E402

HEADS = {"d128": (8, 2, 128), "d64": (4, 4, 64), "mqa": (40, 1, 128), "g256": (256, 1, 64)}


# ---- weights ----

class Weights:
    def __init__(self, segs, heads=(8, 2, 128), seed=1, flags=0, more=0, q_pad=0):
        """segs: per sequence [(start, length), ...]."""
        self.segs, (self.hq, self.hkv, self.d) = segs, heads
        self.ends = [max((s + n for s, n in x), default=0) for x in segs]
        self.lens = [e + more for e in self.ends]
        self.table, self.k, self.v = paged(self.lens, self.hkv, self.d, seed)
        self.rows = sum(n for x in segs for _, n in x)
        g = torch.Generator().manual_seed(seed + 1)
        width = self.hq * self.d + q_pad
        self.q = torch.randn(self.rows, width, generator=g).to(torch.bfloat16).cuda()
        self.scale = self.d ** -0.5
        self.shape = msa.make_shape(len(segs), self.hq, self.hkv, self.d, self.table.shape[1], self.k.shape[0],
                                    self.scale, q_strides=(width, self.d))
        flat = [y for x in segs for y in x]
        indptr = np.cumsum([0] + [len(x) for x in segs])
        self.plan = msa.msa_plan(self.shape, self.lens, indptr, [s for s, _ in flat], [n for _, n in flat], flags=flags)
        self.o = torch.empty(self.rows, self.hq, self.d, dtype=torch.bfloat16, device="cuda")
        self.lse = torch.empty(self.rows, self.hq, device="cuda")
        need = self.plan.info()["workspace_bytes"]
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        msa.msa_forward(self.plan, self.q, self.k, self.v, self.table, self.o, self.lse, ws)
        n = self.table.shape[1] * 16
        self.before = torch.rand(len(segs), self.hkv, n + 5, generator=g).cuda()
        need = msa.msa_kv_weights_workspace(self.plan)
        self.ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda") if need else None

    def run(self, accumulate=True, stream=None, out=None):
        w = self.before.clone() if out is None else out
        msa.msa_kv_weights(self.plan, self.q, self.k, self.table, self.lse, w, self.ws, accumulate, stream=stream)
        return w

    def reference(self):
        G, row = self.hq // self.hkv, 0
        out = torch.zeros(self.before.shape, dtype=torch.float64, device="cuda")
        q = self.q[:, :self.hq * self.d].reshape(-1, self.hq, self.d)
        for b, x in enumerate(self.segs):
            for s, n in x:
                at = torch.arange(s, s + n, device="cuda")
                for h in range(self.hq):
                    k = rows64(self.k, self.table[b], s + n, h // G, False)
                    w = torch.exp((q[row:row + n, h].double() @ k.T) * self.scale - self.lse[row:row + n, h, None].double())
                    w = torch.where(self.lse[row:row + n, h, None] == -float("inf"), 0.0, w)
                    w = torch.where(torch.arange(s + n, device="cuda")[None, :] <= at[:, None], w, 0.0)
                    out[b, h // G, :s + n] += w.sum(0)
                row += n
        return out

    def check(self, w, accumulate=True):
        torch.cuda.synchronize()
        ref = self.reference()
        for b, end in enumerate(self.ends):
            old = self.before[b, :, :end].double() if accumulate else 0.0
            err = (w[b, :, :end].double() - ref[b, :, :end] - old).abs()
            assert (err <= 2.0 ** -17 * ref[b, :, :end] + 2.0 ** -20 * old).all(), (b, err.max().item())
            assert torch.equal(w[b, :, end:], self.before[b, :, end:])  # behind the last row's position: as before


@pytest.mark.parametrize("heads", list(HEADS))
@pytest.mark.parametrize("accumulate", [True, False])
def test_weights_lengths_and_heads(heads, accumulate):
    ends = [1, 2, 15, 16, 17, 31, 33, 63, 64, 65, 100, 255, 256, 257, 300]
    w = Weights([[(0, n)] for n in ends] + [[]] + [[(n - 1, 1)] for n in ends], HEADS[heads], more=3, q_pad=8)
    w.check(w.run(accumulate), accumulate)


@pytest.mark.parametrize("heads", ["d128", "d64", "mqa"])
def test_weights_of_segments(heads):
    r = random.Random(3)
    segs = []
    for L in (900, 513, 64, 2000, 1300):
        a = sorted(r.sample(range(0, L, 7), 6))
        segs.append([(a[0], a[1] - a[0]), (a[2], 1), (a[3], a[4] - a[3]), (L - 2, 2)] if L > 100 else [(L - 1, 1)])
    w = Weights(segs, HEADS[heads])
    w.check(w.run())


@pytest.mark.parametrize("heads", ["d128", "d64"])
def test_weights_of_one_long_row_among_short_ones(heads):
    ends = [3, 40000, 1, 0, 130, 2000] + [65] * 20
    w = Weights([[(n - 1, 1)] if n else [] for n in ends], HEADS[heads], more=1)
    w.check(w.run())


def test_weights_sum_to_the_rows():
    """Each row's weights sum to one: over all keys, rows x heads."""
    w = Weights([[(0, 1500)], [(3000, 1), (3100, 100)]], (32, 8, 128))
    got = w.run(accumulate=False)
    w.check(got, accumulate=False)
    for b, rows in enumerate((1500, 101)):
        total = got[b, :, :w.ends[b]].double().sum(1)
        assert ((total / (rows * 4) - 1).abs() <= 2.0 ** -16).all()


def test_weights_long_decode_and_prompt():
    w = Weights([[(20000, 1)], [(0, 2500)], [(7, 1)]], (16, 2, 128))
    w.check(w.run())


def test_weights_of_rows_without_any_and_odd_values():
    """A row with lse = -inf gives nothing; a key of NaN spoils its own weight alone."""
    w = Weights([[(0, 70)], [(100, 5)]])
    w.lse[3] = -float("inf")
    w.lse[70, 1] = -float("inf")
    w.check(w.run())
    pos = 40
    w.k[w.table[0, pos // 16].long(), 1, pos % 16] = float("nan")
    got = w.run()
    assert torch.isnan(got[0, 1, pos]) and torch.isnan(got).sum().item() == 1


def test_weights_deterministic_on_another_stream_and_in_a_graph():
    w = Weights([[(0, 600)], [(3000, 1)], [(50, 200)]])
    torch.cuda.synchronize()
    a, side = w.run(), torch.cuda.Stream()
    b = w.before.clone()
    torch.cuda.synchronize()
    w.run(stream=side, out=b)
    torch.cuda.synchronize()
    assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    b.copy_(w.before)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        w.run(out=b)
    for _ in range(3):
        b.copy_(w.before)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(a, b)
        assert torch.equal(w.run(), a)


# ---- selection ----

def select64(scores, n, keep, first, recent):
    k = max(0, min(keep, n))
    recent = min(recent, k)
    first = min(first, k - recent)
    window = list(range(first)) + list(range(n - recent, n))
    x = np.where(np.isnan(scores[:n]), -np.inf, scores[:n])[first:n - recent]
    best = np.lexsort((np.arange(len(x)), -x))[:k - first - recent] + first
    return np.sort(np.concatenate([np.array(window, dtype=np.int64), best]))


def check_select(scores, lens, keep, first=4, recent=16, max_keep=None):
    B, H, L = scores.shape
    width = max_keep if max_keep is not None else max(max(keep), 1)
    index = torch.full((B, H, width + 2), -9, dtype=torch.int32, device="cuda")
    count = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    dev = torch.tensor(scores).cuda()
    msa.msa_kv_select(dev, torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor(keep, dtype=torch.int32).cuda(),
                      index[:, :, :width], count, first, recent)
    torch.cuda.synchronize()
    index, count = index.cpu().numpy(), count.cpu().numpy()
    for b in range(B):
        n = max(0, min(lens[b], L))
        k = max(0, min(keep[b], n, width))
        assert count[b] == k
        for h in range(H):
            want = select64(scores[b, h].astype(np.float64), n, k, first, recent)
            assert np.array_equal(index[b, h, :k], want), (b, h)
            assert (index[b, h, k:] == -9).all()


# buffers whose lists are held in 32 or 64 registers a thread, or read again
@pytest.mark.parametrize("L", [70001, 65536, 32769, 32768, 8193])
@pytest.mark.parametrize("values", ["spread", "ties", "equal", "signed", "odd"])
def test_select_lengths(values, L):
    rng = np.random.default_rng(2)
    lens = [0, 1, 2, 20, 21, 63, 64, 65, 1000, 1023, 1024, 1025, 2049, 5000, L - 1, -3, 99999]
    x = rng.random((len(lens), 2, L), dtype=np.float32) ** 4 * 8
    if values == "ties":
        x = np.round(x * 8) / 8
    elif values == "equal":
        x[:] = 0.25
    elif values == "signed":
        x = (rng.standard_normal(x.shape) * 10).astype(np.float32)
        x[:, :, ::3] = 0.0
        x[:, :, 1::3] = -0.0
    elif values == "odd":
        x[:, :, ::5] = np.nan
        x[:, :, 1::7] = -np.inf
        x[:, :, 2::11] = np.inf
        x[:, :, 3::5] = 1e-42
    keep = [3, 1, 1, 20, 20, 30, 64, 10, 500, 1, 1024, 700, 0, 4999, L // 7 * 3, 5, L]
    check_select(x.astype(np.float32), lens, keep)


@pytest.mark.parametrize("first,recent", [(0, 0), (0, 50), (50, 0), (1000, 1000), (3, 2 ** 31 - 1), (2 ** 31 - 1, 3)])
def test_select_windows(first, recent):
    rng = np.random.default_rng(3)
    x = rng.random((4, 3, 900), dtype=np.float32)
    check_select(x, [900, 100, 64, 7], [90, 99, 64, 200], first, recent)


def test_select_more_to_keep_than_the_list_holds():
    rng = np.random.default_rng(4)
    check_select(rng.random((3, 1, 500), dtype=np.float32), [500, 300, 40], [400, 2 ** 31 - 1, -7], 4, 8, max_keep=60)


def test_select_in_a_graph_and_on_another_stream():
    g = torch.Generator().manual_seed(6)
    x = torch.rand(3, 4, 3000, generator=g).cuda()
    n, k = torch.tensor([3000, 17, 1200], dtype=torch.int32).cuda(), torch.tensor([900, 30, 1], dtype=torch.int32).cuda()
    out = [torch.full((3, 4, 900), -1, dtype=torch.int32, device="cuda") for _ in range(3)]
    cnt = torch.empty(3, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    msa.msa_kv_select(x, n, k, out[0], cnt, 4, 8, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        msa.msa_kv_select(x, n, k, out[1], cnt, 4, 8)
    for _ in range(3):
        x.copy_(torch.rand(3, 4, 3000, generator=g))
        out[1].fill_(-1)
        out[2].fill_(-1)
        graph.replay()
        msa.msa_kv_select(x, n, k, out[2], cnt, 4, 8)
        torch.cuda.synchronize()
        assert torch.equal(out[1], out[2])
        for b in range(3):
            want = select64(x[b, 2].cpu().numpy().astype(np.float64), int(n[b]), int(k[b]), 4, 8)
            assert np.array_equal(out[1][b, 2, :len(want)].cpu().numpy(), want)


def test_select_many_and_strided_lists():
    rng = np.random.default_rng(5)
    B, H, L = 40, 8, 777
    lens = [int(v) for v in rng.integers(1, L, B)]
    keep = [int(v) for v in rng.integers(1, L, B)]
    x = rng.random((B, H, L), dtype=np.float32)
    check_select(x, lens, keep)
    big = torch.rand(B, 2 * H, L + 3, device="cuda")
    view = big[:, ::2, 1:L + 1]
    out = torch.full((B, H, L), -1, dtype=torch.int32, device="cuda")
    cnt = torch.empty(B, dtype=torch.int32, device="cuda")
    n, k = torch.tensor(lens, dtype=torch.int32).cuda(), torch.tensor(keep, dtype=torch.int32).cuda()
    msa.msa_kv_select(view, n, k, out, cnt, 2, 5)
    for b in (0, 7, 39):
        want = select64(view[b, 3].cpu().numpy().astype(np.float64), lens[b], keep[b], 2, 5)
        assert np.array_equal(out[b, 3, :len(want)].cpu().numpy(), want)


# ---- compaction ----

def compact_ref(k, v, table, base, lists, counts, cap):
    """Element by element on the host, from copies."""
    k0, v0, table = k.clone(), v.clone(), table.tolist()
    nblk, H = k.shape[0], k.shape[1]

    def place(b, pos):
        if not 0 <= pos < cap:
            return None
        blk = table[b][pos // 16]
        return (blk, pos % 16) if 0 <= blk < nblk else None

    for b, n in enumerate(counts):
        for h in range(H):
            idx = lists[b][h]
            for i in range(min(max(n, 0), len(idx))):
                s, d = place(b, base[b] + idx[i]), place(b, base[b] + i)
                if s and d:
                    k[d[0], h, d[1]] = k0[s[0], h, s[1]]
                    v[d[0], h, :, d[1]] = v0[s[0], h, :, s[1]]
    return k, v


def check_compact(lens, base, counts, lists, heads=(2, 128), shared=False, spoil=(), seed=1, strides=False,
                  swap=()):
    hkv, d = heads
    table, k, v = paged(lens, hkv, d, seed)
    for b, i, blk in spoil:
        table[b, i] = blk
    for b, i, blk in swap:  # physical block blk at logical block i, its owner gets the other one
        old = table[b, i].clone()
        table[table == blk] = old
        table[b, i] = blk
    kw = {}
    if strides:  # heads outermost in the block, padded rows
        kb = torch.randn(k.shape[0], 16, hkv, d + 8).to(torch.bfloat16).cuda()
        kb[..., :d] = k.permute(0, 2, 1, 3)
        k = kb.permute(0, 2, 1, 3)[..., :d]
        vb = torch.randn(v.shape[0], hkv, d, 24).to(torch.bfloat16).cuda()
        vb[..., :16] = v
        v = vb[..., :16]
        kw = dict(k_strides=(k.stride(0), k.stride(1), k.stride(2)), v_strides=(v.stride(0), v.stride(1), v.stride(2)))
    shape = msa.make_shape(len(lens), hkv, hkv, d, table.shape[1], k.shape[0], 1.0, **kw)
    width = max(len(x) for row in lists for x in row)
    index = torch.full((len(lens), hkv, width), 1 << 30, dtype=torch.int32)
    for b, row in enumerate(lists):
        for h, x in enumerate(row):
            index[b, h, :len(x)] = torch.tensor(x, dtype=torch.int32)
    want_k, want_v = compact_ref(k.cpu(), v.cpu(), table.cpu(), base, lists, counts, table.shape[1] * 16)
    dev = index[:, 0].contiguous().cuda() if shared else index.cuda()
    b_dev = torch.tensor(base, dtype=torch.int32).cuda() if any(base) else None
    msa.msa_kv_compact(shape, b_dev, dev, torch.tensor(counts, dtype=torch.int32).cuda(), table, k, v)
    torch.cuda.synchronize()
    assert torch.equal(k.cpu().contiguous().view(torch.int16), want_k.contiguous().view(torch.int16))
    assert torch.equal(v.cpu().contiguous().view(torch.int16), want_v.contiguous().view(torch.int16))


def pick(r, n, k):
    return sorted(r.sample(range(n), k))


@pytest.mark.parametrize("heads", [(2, 128), (3, 64)])
@pytest.mark.parametrize("shared", [True, False])
def test_compact_lists(heads, shared):
    r = random.Random(6)
    lens = [1, 2, 16, 17, 63, 64, 65, 130, 300, 1000, 700]
    counts = [1, 1, 8, 17, 1, 63, 40, 129, 7, 500, 0]
    lists = []
    for n, c in zip(lens, counts):
        one = pick(r, n, c)
        lists.append([one if shared else pick(r, n, c) for _ in range(heads[0])])
    check_compact(lens, [0] * len(lens), counts, lists, heads, shared)


@pytest.mark.parametrize("strides", [False, True])
def test_compact_behind_a_base(strides):
    """The accepted slots of trees: lists relative to any position, moves inside and across blocks."""
    r = random.Random(7)
    base = [0, 1, 5, 7, 8, 9, 15, 16, 23, 100, 333]
    lists, counts = [], []
    for i, _ in enumerate(base):
        c = (i * 5) % 14 + 1
        lists.append([[0] + sorted(r.sample(range(1, 40), c - 1))] * 2)
        counts.append(c)
    check_compact([b + 40 for b in base], base, counts, lists, shared=True, strides=strides)


def test_compact_patterns():
    n = 600
    for idx in (list(range(n)), list(range(1, n)), list(range(0, n, 2)), list(range(n - 64, n)), [n - 1],
                list(range(16, n)), list(range(8, n)), list(range(0, 300)) + list(range(316, n)),
                [0, 1, 2, 3] + list(range(64, n, 3))):
        check_compact([n], [0], [len(idx)], [[idx, idx]])
        check_compact([n + 11], [11], [len(idx)], [[idx, idx]])


def test_compact_long():
    r = random.Random(8)
    lens = [9000, 5000]
    counts = [4500, 4999]
    check_compact(lens, [0, 0], counts, [[pick(r, n, c) for _ in range(2)] for n, c in zip(lens, counts)], (2, 64))


def test_compact_with_any_block_anywhere():
    """Physical block 0 (and every other) as a source behind kept places and behind skipped moves, at every block of a
    sequence."""
    r = random.Random(10)
    for at in range(12):
        lens = [192, 192]
        idx = list(range(5)) + pick(r, 187, 150)
        idx = sorted(set(x + 5 if i >= 5 else x for i, x in enumerate(idx)))
        table_order = [(0, at, 0)]
        check_compact(lens, [0, 3], [len(idx)] * 2, [[idx, idx]] * 2, shared=True, swap=table_order)


@pytest.mark.parametrize("part", [0.02, 0.1, 0.3, 0.6, 0.9, 0.99])
@pytest.mark.parametrize("first", [0, 4, 70])
def test_compact_parts_of_a_list(part, first):
    """Few and many kept tokens a block, runs whose places all move and runs where some stay where they are."""
    r = random.Random(int(part * 100) + first)
    lens, base = [3001, 40, 6000, 130], [0, 5, 16, 39]
    counts = [max(1, int(n * part)) for n in lens]
    lists = [[(sorted(set(range(min(first, n))) | set(r.sample(range(n), k)))[:k]) for _ in range(2)]
             for n, k in zip(lens, counts)]
    check_compact([n + b for n, b in zip(lens, base)], base, counts, lists, seed=first + 2)


def test_compact_skips_what_lies_outside():
    """Blocks outside the cache, positions past the table, counts past the list."""
    idx = list(range(3, 80, 2))
    lens = [90, 90, 90]
    check_compact(lens, [0, 0, 0], [len(idx), 1000, -4], [[idx, idx]] * 3,
                  spoil=[(0, 1, -1), (0, 4, 1 << 30), (1, 0, -5)])
    far = [1, 50, 95, 96, 97, 200]
    check_compact([90], [0], [len(far)], [[far, far]])
    check_compact([90], [2 ** 31 - 1], [len(far)], [[far, far]])
    check_compact([90], [-20], [len(idx)], [[idx, idx]])


def test_compact_in_a_graph():
    r = random.Random(9)
    table, k, v = paged([500], 2, 128, 1)
    shape = msa.make_shape(1, 2, 2, 128, table.shape[1], k.shape[0], 1.0)
    idx = torch.tensor([pick(r, 500, 200)], dtype=torch.int32).cuda()
    cnt = torch.tensor([200], dtype=torch.int32).cuda()
    a, b = k.clone(), v.clone()
    msa.msa_kv_compact(shape, None, idx, cnt, table, a, b)
    k2, v2 = k.clone(), v.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        msa.msa_kv_compact(shape, None, idx, cnt, table, k2, v2)
    for _ in range(3):
        k2.copy_(k)
        v2.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(k2.view(torch.int16), a.view(torch.int16))
        assert torch.equal(v2.view(torch.int16), b.view(torch.int16))
