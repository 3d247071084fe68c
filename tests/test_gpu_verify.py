"""Verification of drafted trees (msa_tree_verify) against a plain walk in 64
bits that holds every residual in full (GPU only).  Outputs are whole numbers
and have to be equal; drawn inputs keep no test and no drawn token within 1e-12 of
a border (checked in the walk), where 64-bit sums of another order could differ.
"""
import random

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

import paper_2606_02964_amd as msa  # noqa: E402
from tree_ref import random_parents  # noqa: E402

NEAR = 1e-12


def clean(x):
    x = np.asarray(x, dtype=np.float64).copy()
    x[~np.isfinite(x) | (x < 0)] = 0.0
    return x


def walk64(parents, tokens, target, draft, u_accept, u_sample):
    """(path, next token, whether a decision was near a border)."""
    node, path, near = 0, [0], False
    V = target.shape[1]

    def below(a, b):
        nonlocal near
        near |= abs(a - b) < NEAR * max(abs(a), abs(b)) and a != b
        return a < b

    while True:
        p = clean(target[node])
        r, mass, stay = p.copy(), 1.0, None
        for i, up in enumerate(parents):
            if up != node or i <= node:
                continue
            x = tokens[i]
            ok = 0 <= x < V
            if draft is not None:
                q = clean(draft[node])
                if mass > 0 and ok and below(float(u_accept[i]) * q[x] * mass, r[x]):
                    stay = i
                    break
                r = np.maximum(r / mass - q, 0.0) if mass > 0 else r * 0.0
                mass = r.sum()
            else:
                if ok and below(float(u_accept[i]) * mass, r[x]):
                    stay = i
                    break
                if ok:
                    mass -= r[x]
                    r[x] = 0.0
        if stay is None:
            break
        node = stay
        path.append(node)
    c = np.cumsum(r)
    if not c[-1] > 0:
        c = np.cumsum(p)
    if not c[-1] > 0:
        return path, -1, near
    u = float(u_sample)
    u = min(max(u, 0.0), 1.0 - 2.0 ** -24) if u == u else 0.0
    x = u * c[-1]
    past = np.nonzero(c > x)[0]
    if u > 0:
        near |= bool(np.abs(c - x).min() < NEAR * c[-1])
    t = int(past[0]) if len(past) else int(np.nonzero(np.diff(c, prepend=0.0) > 0)[0][-1])
    return path, t, near


class Drafts:
    def __init__(self, trees, vocab, kind="drawn", dtype=torch.float32, seed=1, noise=0.7, pad=0, sharp=3.0):
        g = torch.Generator().manual_seed(seed)
        n = sum(len(t) for t in trees)
        self.trees, self.vocab, self.dtype = trees, vocab, dtype
        logits = sharp * torch.randn(n, vocab, generator=g)
        self.target = self._rows(torch.softmax(logits, 1), pad)
        self.draft = self._rows(torch.softmax(logits + noise * torch.randn(n, vocab, generator=g), 1), pad)
        self.parents = torch.tensor([p for t in trees for p in t], dtype=torch.int32)
        self.tokens = torch.zeros(n, dtype=torch.int32)
        at = 0
        for t in trees:
            for i, p in enumerate(t):
                if not 0 <= p < i:
                    continue
                q = self.draft[at + p, :vocab].float()
                if kind == "best":
                    rank = sum(1 for y in t[:i] if y == p)
                    self.tokens[at + i] = torch.topk(q, min(vocab, rank + 1)).indices[-1]
                else:
                    self.tokens[at + i] = torch.multinomial(q, 1, generator=g)[0]
            at += len(t)
        if kind == "best":
            self.draft = None
        self.u_accept = torch.rand(n, generator=g)
        self.u_sample = torch.rand(len(trees), generator=g)

    def _rows(self, x, pad):
        out = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=self.dtype)
        out[:, :x.shape[1]] = x.to(self.dtype)
        return out

    def run(self, graph=False):
        t = self.trees
        m = [len(x) for x in t]
        shape = msa.make_shape(len(t), 8, 8, 128, -(-max(m) // 16), sum(-(-x // 16) for x in m), 1.0)
        self.plan = plan = msa.msa_plan_tree(shape, m, list(range(len(m) + 1)), [0] * len(m), m)
        dev = {k: None if v is None else v.cuda() for k, v in vars(self).items() if isinstance(v, torch.Tensor) or v is None}
        path = torch.full((len(t), max(m) + 2), 77, dtype=torch.int32, device="cuda")
        length = torch.full((len(t),), 77, dtype=torch.int32, device="cuda")
        token = torch.full((len(t),), 77, dtype=torch.int32, device="cuda")
        need = msa.msa_tree_verify_workspace(plan, self.vocab)
        ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
        target = dev["target"][:, :self.vocab]
        draft = dev.get("draft")
        draft = None if draft is None else draft[:, :self.vocab]
        call = lambda: msa.msa_tree_verify(plan, target, dev["tokens"], dev["parents"], dev["u_accept"],  # noqa: E731
                                           dev["u_sample"], path, length, token, draft, ws)
        call()
        if graph:
            torch.cuda.synchronize()
            first = (path.clone(), length.clone(), token.clone())
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                call()
            for _ in range(3):
                for x in (path, length, token):
                    x.fill_(77)
                g.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(first, (path, length, token)))
        torch.cuda.synchronize()
        return path.cpu().numpy(), length.cpu().numpy(), token.cpu().numpy()

    def check(self, **kw):
        path, length, token = self.run(**kw)
        at, most, near = 0, max(len(t) for t in self.trees), 0
        target = self.target[:, :self.vocab].double().numpy()
        draft = None if self.draft is None else self.draft[:, :self.vocab].double().numpy()
        for t, parents in enumerate(self.trees):
            n = len(parents)
            want, nxt, close = walk64(parents, self.tokens[at:at + n].tolist(), target[at:at + n],
                                      None if draft is None else draft[at:at + n], self.u_accept[at:at + n].numpy(),
                                      self.u_sample[t].numpy())
            at += n
            if close:
                near += 1
                continue
            got = path[t]
            assert length[t] == len(want) and got[:len(want)].tolist() == want, (t, got, want)
            assert (got[len(want):most] == -1).all() and (got[most:] == 77).all()
            assert token[t] == nxt, (t, token[t], nxt)
        assert near <= len(self.trees) // 50, near


def trees_of(seed, sizes, kind):
    r = random.Random(seed)
    return [random_parents(r, m, kind) for m in sizes]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("kind", ["drawn", "best"])
@pytest.mark.parametrize("shape", ["chain", "tree", "star", "forest"])
def test_shapes_and_types(shape, kind, dtype):
    Drafts(trees_of(1, [1, 2, 3, 8, 8, 16, 33, 64, 65, 5, 90], shape), 997, kind, dtype, pad=3).check()


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 64, 255, 511, 513, 2047, 4099, 8192, 8193, 32000, 32768, 32769, 50257])
@pytest.mark.parametrize("kind", ["drawn", "best"])
def test_vocabularies(vocab, kind):
    Drafts(trees_of(2, [6, 9, 1, 4], "tree"), vocab, kind).check()


def test_large_trees():
    Drafts(trees_of(3, [1024, 700], "tree"), 300, "drawn", sharp=1.0).check()
    Drafts(trees_of(3, [1024, 700], "star"), 300, "drawn", noise=2.0).check()
    Drafts(trees_of(3, [1024, 130], "star"), 3000, "best").check()


def test_a_vocabulary_in_few_and_in_many_chunks():
    Drafts(trees_of(4, [2], "chain"), 151937, "drawn", noise=3.0).check()
    Drafts(trees_of(5, [2] * 600, "chain"), 5003, "drawn", noise=2.0).check()
    d = Drafts(trees_of(6, [1] * 1500, "chain"), 3001, "drawn")
    d.check()
    Drafts(trees_of(6, [1] * 700, "chain"), 33003, "best").check()  # workgroups that take several cells each


@pytest.mark.parametrize("vocab", [2500, 40000])
@pytest.mark.parametrize("kind", ["drawn", "best"])
def test_graph_replays(vocab, kind):
    Drafts(trees_of(7, [8] * 6, "tree"), vocab, kind).check(graph=True)


def test_ends_of_the_random_numbers():
    d = Drafts(trees_of(8, [4] * 12, "tree"), 500, "drawn")
    u = [0.0, 1.0 - 2.0 ** -24, 1.0, 2.0, -1.0, float("nan"), float("inf"), 0.5, 2.0 ** -30, 0.0, 1.0, 0.25]
    d.u_sample = torch.tensor(u)
    d.u_accept[::3] = 0.0
    d.u_accept[1::3] = 1.0 - 2.0 ** -24
    d.check()


@pytest.mark.parametrize("vocab", [203, 40203])
def test_odd_probabilities_and_tokens(vocab):
    """Zeros, negatives, NaN and infinities count as 0; a token outside the vocabulary never stays; equal rows always
    accept, and a residual without mass falls back to the row."""
    for kind in ("drawn", "best"):
        d = Drafts(trees_of(9, [7] * 9, "star"), vocab, kind)
        n = 7
        d.target[0, ::2] = 0.0                         # a row with zeros
        d.target[n, ::3] = float("nan")
        d.target[n, 1::3] = -1.0
        d.target[2 * n, 5] = float("inf")
        d.target[3 * n:4 * n] = 0.0                    # nothing at all: -1
        d.target[4 * n, :] = 0.0
        d.target[4 * n, 17] = 1.0                      # one token
        d.tokens[5 * n + 1] = vocab
        d.tokens[5 * n + 2] = -1
        d.tokens[5 * n + 3] = 1 << 30
        d.tokens[6 * n + 1:7 * n] = d.tokens[6 * n + 1]  # one token six times
        if d.draft is not None:
            d.draft[7 * n:8 * n] = d.target[7 * n:8 * n]
            d.tokens[8 * n + 1:9 * n] = -5               # tests that fail on a residual without mass
            d.draft[8 * n:9 * n] = d.target[8 * n:9 * n]
        d.check()


@pytest.mark.parametrize("vocab,cell", [(600, 8), (40000, 8), (40000, 512), (30000, 512)])
def test_a_drawn_token_has_weight(vocab, cell):
    """Sums whose rounding depends on their order: e + e + 1 + 0 is 1 or 1 + 2 e, with e = 2^-53, and half the total
    lies between.  Cells of 8 entries are a lane's, of 512 a wave's."""
    row = torch.zeros(1, vocab)
    row[0, 0] = row[0, cell] = 2.0 ** -53
    row[0, 2 * cell] = row[0, 4 * cell] = 1.0
    d = Drafts([[-1]], vocab)
    d.target, d.draft, d.u_sample = row, None, torch.tensor([0.5])
    _, _, token = d.run()
    assert int(token[0]) in (2 * cell, 4 * cell)


def test_tokens_follow_the_target():
    """First kept token of 40000 one-level trees of three drafts, against the target's probabilities: each frequency
    within 5 standard deviations, and the drafts' own distribution is not."""
    n, V = 40000, 6
    g = torch.Generator().manual_seed(1)
    p = torch.tensor([0.40, 0.05, 0.25, 0.0, 0.10, 0.20])
    q = torch.tensor([0.10, 0.30, 0.05, 0.15, 0.30, 0.10])
    d = Drafts([[-1, 0, 0, 0]] * 2, V)
    d.trees = [[-1, 0, 0, 0]] * n
    d.parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32).repeat(n)
    d.target, d.draft = p.repeat(4 * n, 1), q.repeat(4 * n, 1)
    d.tokens = torch.multinomial(q.repeat(1, 1), 4 * n, replacement=True, generator=g)[0].to(torch.int32)
    d.u_accept, d.u_sample = torch.rand(4 * n, generator=g), torch.rand(n, generator=g)
    path, length, token = d.run()
    first = np.where(length > 1, d.tokens.numpy().reshape(n, 4)[np.arange(n), np.maximum(path[:, 1], 0)], token)
    freq = np.bincount(first, minlength=V) / n
    sd = np.sqrt(p.numpy() * (1 - p.numpy()) / n)
    assert (np.abs(freq - p.numpy()) <= 5 * sd).all(), freq
    assert (length > 1).mean() > 0.6
    d.draft = None  # best drafts: tokens 0, 1, 4 everywhere
    d.tokens = torch.tensor([0, 0, 1, 4], dtype=torch.int32).repeat(n)
    path, length, token = d.run()
    first = np.where(length > 1, d.tokens.numpy().reshape(n, 4)[np.arange(n), np.maximum(path[:, 1], 0)], token)
    freq = np.bincount(first, minlength=V) / n
    assert (np.abs(freq - p.numpy()) <= 5 * sd).all(), freq
    assert abs((length > 1).mean() - 0.55) < 0.0125
