"""The speculative-decoding and cache-reduction operators' measured calls.

A case is one call of an operator as a serving step makes it, with the plan,
the workspace and the buffers that such a program keeps from step to step:

* ``tree``: attention of trees of drafted tokens over the paged cache, alone
  ("forward"), after the write of the drafted tokens' K/V ("layer"), or after
  the ancestor mask and that write ("step", the first layer of a step);
* ``verify``: which drafted tokens stay, and the token that follows them;
* ``weights``: the attention weight each cached key receives, added up;
* ``select``: the positions a reduced cache keeps;
* ``compact``: the kept positions' K/V moved to the front, after a verified
  tree ("commit") or a reduction of the cache ("evict").

Sizes are generic: the head layouts of this repository's workloads, contexts
from tens of tokens to 64K, trees of 2 to 128 slots, vocabularies of 1K to
150K.  A case's layout depends on its fields only, its values and the
placement of its cache blocks on the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
BS = 16  # tokens of a cache block

# (query heads, KV heads, head_dim): an 8B and a 70B layer, one tensor-parallel
# rank of each, and heads without grouping at the smaller head dimension
HEADS = ((32, 8, 128), (64, 8, 128), (8, 2, 128), (16, 2, 128), (16, 16, 64), (4, 4, 64))


def listed():
    def tree(name, call, seqs, ctx, slots, heads=(32, 8, 128), kind="tree", chunk=0, lse=False):
        return dict(name=name, op="tree", call=call, seqs=seqs, ctx=ctx, slots=slots, kind=kind, chunk=chunk,
                    hq=heads[0], hkv=heads[1], d=heads[2], lse=lse, layout_seed=3)

    def verify(name, trees, slots, vocab, kind, dtype):
        return dict(name=name, op="verify", trees=trees, slots=slots, vocab=vocab, kind=kind, dtype=dtype, layout_seed=3)

    def weights(name, layout, seqs, ctx, new, heads=(32, 8, 128)):
        return dict(name=name, op="weights", layout=layout, seqs=seqs, ctx=ctx, new=new, hq=heads[0], hkv=heads[1],
                    d=heads[2], layout_seed=3)

    def select(name, seqs, lists, ctx, part, ties=False):
        return dict(name=name, op="select", seqs=seqs, lists=lists, ctx=ctx, part=part, ties=ties, layout_seed=3)

    def compact(name, call, seqs, ctx, slots, part, shared, heads=(32, 8, 128)):
        return dict(name=name, op="compact", call=call, seqs=seqs, ctx=ctx, slots=slots, part=part, shared=shared,
                    hkv=heads[1], d=heads[2], layout_seed=3)

    return [
        # the smallest call: a first step's mask, cache write and attention, five slots over 200 tokens
        tree("tree_tiny", "step", 1, 200, 5, heads=(4, 4, 64), lse=True),
        # one user with a wide tree over 8K tokens of context
        tree("tree_one", "forward", 1, 8190, 61),
        # a serving batch of 16-slot trees, with their cache write
        tree("tree_batch", "layer", 48, 6000, 16),
        # wide trees of a 70B layer over long contexts, every fourth sequence a prefill chunk: the largest call
        tree("tree_long", "forward", 16, 30001, 64, heads=(64, 8, 128), chunk=128, lse=True),
        # a batch of drafted chains of up to 7 tokens, each drawn from a draft model
        verify("verify_chain", 32, 8, 131072, "chain", "float32"),
        # one wide tree of the draft model's best tokens
        verify("verify_best", 1, 61, 32000, "best", "float32"),
        # a decoding batch adds up its weights at every step
        weights("weights_decode", "decode", 64, 8000, 1),
        # prompts add theirs up once
        weights("weights_prompt", "prompt", 3, 4099, 0),
        # one user's cache to a quarter of its positions, one list for all heads
        select("select_one", 1, 1, 9001, 0.25),
        # a batch's caches to a half, a list for each head
        select("select_batch", 32, 8, 16384, 0.5),
        # the accepted slots of a batch of trees
        compact("compact_commit", "commit", 48, 6000, 16, 0.0, True),
        # a batch's caches to a half, each head its own positions
        compact("compact_evict", "evict", 16, 16384, 0, 0.5, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, sizes spread over their logarithm, odd
    ones among them, no larger than the largest listed case."""
    while True:
        op = rng.choice(("tree", "tree", "verify", "weights", "select", "compact"))
        hq, hkv, d = rng.choice(HEADS)
        case = dict(op=op, layout_seed=rng.randrange(1 << 20))
        if op == "tree":
            case.update(call=rng.choice(("forward", "layer", "step")), seqs=_log_int(rng, 1, 48),
                        ctx=_log_int(rng, 16, 30000), slots=_log_int(rng, 2, 128), kind=rng.choice(("tree", "chain")),
                        chunk=rng.choice((0, 0, _log_int(rng, 1, 200))), hq=hq, hkv=hkv, d=d, lse=rng.random() < 0.5)
            cost = case["seqs"] * hq * max(case["slots"], case["chunk"]) * (case["ctx"] + 128)
            most = 16 * 64 * 128 * 30001
        elif op == "verify":
            case.update(trees=_log_int(rng, 1, 64), slots=_log_int(rng, 2, 64), vocab=_log_int(rng, 1000, 150000),
                        kind=rng.choice(("chain", "best", "drawn")), dtype=rng.choice(("float32", "float32", "bfloat16")))
            cost, most = case["trees"] * case["slots"] * case["vocab"], 32 * 8 * 131072
        elif op == "weights":
            layout = rng.choice(("decode", "prompt", "chunks"))
            ctx = _log_int(rng, 16, 16384 if layout == "decode" else 6000)
            case.update(layout=layout, seqs=_log_int(rng, 1, 96 if layout == "decode" else 8), ctx=ctx,
                        new=1 if layout == "decode" else min(ctx, _log_int(rng, 2, 1024)), hq=hq, hkv=hkv, d=d)
            rows = {"decode": 1, "prompt": ctx, "chunks": 2 * case["new"]}[layout]
            cost, most = case["seqs"] * hq * rows * ctx, 3 * 32 * 4099 * 4099
        elif op == "select":
            case.update(seqs=_log_int(rng, 1, 32), lists=rng.choice((1, 2, 8)), ctx=_log_int(rng, 30, 65536),
                        part=round(rng.uniform(0.05, 0.95), 3), ties=rng.random() < 0.5)
            cost, most = case["seqs"] * case["lists"] * case["ctx"], 32 * 8 * 16384
        else:
            call = rng.choice(("commit", "evict"))
            case.update(call=call, seqs=_log_int(rng, 1, 48 if call == "commit" else 16),
                        ctx=_log_int(rng, 16, 16384), slots=_log_int(rng, 2, 64) if call == "commit" else 0,
                        part=0.0 if call == "commit" else round(rng.uniform(0.05, 0.95), 3),
                        shared=call == "commit" or rng.random() < 0.5, hkv=hkv, d=d)
            cost, most = case["seqs"] * hkv * d * (case["ctx"] + 128), 16 * 8 * 128 * 16512 * 3
        if cost <= most:
            return case


# ---- layouts: plain host numbers from a case's fields ----

def _lengths(r, n, top):
    return [top if n == 1 else r.randint(max(1, top // 8), top) for _ in range(n)]


def _parents(r, m, kind):
    """Parent slot of each slot of a tree, -1 for the root (slot 0)."""
    if kind == "chain":
        return list(range(-1, m - 1))
    return [-1] + [r.randint(max(0, (i - 1) // 3 - 1), i - 1) for i in range(1, m)]


def _tree_layout(case):
    """Per sequence: the context before its new rows, their number, and the
    tree's parents (None for a causal chunk)."""
    r = random.Random(case["layout_seed"])
    ctx = _lengths(r, case["seqs"], case["ctx"])
    out = []
    for b, c in enumerate(ctx):
        if case["chunk"] and b % 4 == 3:
            out.append((c, case["chunk"], None))
        else:
            m = case["slots"] if case["seqs"] == 1 else r.randint(max(2, case["slots"] // 2), case["slots"])
            out.append((c, m, _parents(r, m, case["kind"])))
    return out


def _weights_layout(case):
    """Context length and (start, length) query segments of each sequence."""
    r = random.Random(case["layout_seed"])
    out = []
    for L in _lengths(r, case["seqs"], case["ctx"]):
        if case["layout"] == "decode":
            segs = [(L - 1, 1)]
        elif case["layout"] == "prompt":
            segs = [(0, L)]
        else:  # a recomputed chunk earlier on and the new tokens at the end
            n = min(case["new"], L)
            first = min(n, max(0, (L - n) // 2))
            segs = ([(L // 5, first)] if first and L // 5 + first <= L - n else []) + [(L - n, n)]
        out.append((L, segs))
    return out


def _verify_layout(case):
    r = random.Random(case["layout_seed"])
    sizes = [case["slots"] if case["trees"] == 1 else r.randint(max(2, case["slots"] // 2), case["slots"])
             for _ in range(case["trees"])]
    return [_parents(r, m, "chain" if case["kind"] == "chain" else "tree") for m in sizes]


def _depths(parents):
    out = []
    for p in parents:
        out.append(0 if p < 0 else out[p] + 1)
    return out


def work(case):
    op = case["op"]
    if op == "tree":
        nbytes = flops = 0
        for c, m, par in _tree_layout(case):
            nbytes += 4 * m * case["hq"] * case["d"] + (c + m) * case["hkv"] * case["d"] * 4
            nbytes += (8 * ((m + 63) // 64) * m if par else 0) + (4 * m * case["hq"] if case["lse"] else 0)
            nbytes += 4 * m * case["hkv"] * case["d"] * 2 if case["call"] != "forward" else 0
            own_keys = sum(x + 1 for x in _depths(par)) if par else m * (m + 1) // 2
            flops += 4 * case["d"] * case["hq"] * (m * c + own_keys)
        return {"bytes": nbytes, "flops": flops}
    if op == "verify":
        # each draft's two probabilities, and the target's and the draft's row that the next token is drawn from
        size = 2 if case["dtype"] == "bfloat16" else 4
        rows = 1 if case["kind"] == "best" else 2
        slots = sum(len(p) for p in _verify_layout(case))
        return {"bytes": slots * (16 + rows * size) + case["trees"] * (case["vocab"] * rows * size + 16),
                "flops": 3 * case["trees"] * case["vocab"]}
    if op == "weights":
        nbytes = flops = 0
        for L, segs in _weights_layout(case):
            rows = sum(n for _, n in segs)
            end = segs[-1][0] + segs[-1][1]
            nbytes += rows * case["hq"] * (2 * case["d"] + 4) + end * case["hkv"] * (2 * case["d"] + 8)
            flops += 2 * case["d"] * case["hq"] * sum(n * a + n * (n + 1) // 2 for a, n in segs)
        return {"bytes": nbytes, "flops": flops}
    r = random.Random(case["layout_seed"])
    if op == "select":
        lens = _lengths(r, case["seqs"], case["ctx"])
        return {"bytes": sum(case["lists"] * 4 * (L + min(L, int(L * case["part"]) + 8)) for L in lens),
                "flops": sum(case["lists"] * L for L in lens)}
    lens = _lengths(r, case["seqs"], case["ctx"])
    if case["call"] == "commit":
        moved = sum(max(1, case["slots"] // 4) for _ in lens)
    else:
        moved = sum(int(L * case["part"]) + 1 for L in lens)
    return {"bytes": moved * case["hkv"] * case["d"] * 8, "flops": 0}


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=DEV).normal_(generator=g)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _cache(g, lens, hkv, d):
    """Scattered cache blocks for sequences of these lengths."""
    counts = [-(-L // BS) for L in lens]
    n, most = sum(counts), max(counts)
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(most, device=DEV)[None, :] < _ints(counts)[:, None]] = \
        torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    return table, _normal(g, n, hkv, BS, d), _normal(g, n, hkv, d, BS)


def _padded(counts):
    """Packed row of each (sequence, place), and which places hold one."""
    start = torch.cumsum(_ints([0] + list(counts), torch.int64), 0)
    place = torch.arange(max(counts), device=DEV)
    valid = place[None, :] < _ints(counts)[:, None]
    return torch.where(valid, start[:-1, None] + place[None, :], 0), valid


def prepare(case, seed):
    s = {"case": case}
    {"tree": _prepare_tree, "verify": _prepare_verify, "weights": _prepare_weights, "select": _prepare_select,
     "compact": _prepare_compact}[case["op"]](case, _generator(seed), s)
    return s


def _prepare_tree(case, g, s):
    lay = _tree_layout(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens = [c + m for c, m, _ in lay]
    rows = sum(m for _, m, _ in lay)
    s["table"], s["k_cache"], s["v_cache"] = _cache(g, lens, hkv, d)
    s["q"] = _normal(g, rows, hq, d)
    kv = _normal(g, rows, 2 * hkv, d)  # one fused projection's output, as a model has it
    s["k_new"], s["v_new"] = kv[:, :hkv], kv[:, hkv:]
    s["o"] = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.empty(rows, hq, dtype=torch.float32, device=DEV) if case["lse"] else None
    # the trees: a parent for each slot, slots counted from the tree's own root
    trees = [p for _, _, p in lay if p is not None]
    s["parents"] = _ints([x for p in trees for x in p])
    words = -(-max(len(p) for p in trees) // 64) if trees else 1
    s["mask"] = torch.zeros(len(s["parents"]), words, dtype=torch.int64, device=DEV)
    s["tree_rows"], s["tree_valid"] = _padded([len(p) for p in trees])
    if case["call"] != "step":
        s["mask"].copy_(_ancestors(s))
    # where each row stands
    s["start"] = _ints([c for c, _, _ in lay], torch.int64)
    s["rows"], s["valid"] = _padded([m for _, m, _ in lay])
    at, n = [], 0
    for _, m, p in lay:
        at += list(range(n, n + m)) if p is not None else [-1] * m
        n += m if p is not None else 0
    s["mask_row"] = _ints(at, torch.int64)
    s["scale"] = d ** -0.5
    if own:
        import paper_2606_02964_amd as msa
        shape = msa.make_shape(len(lay), hq, hkv, d, s["table"].shape[1], s["k_cache"].shape[0], s["scale"])
        s["plan"] = msa.msa_plan_tree(shape, lens, list(range(len(lay) + 1)), [c for c, _, _ in lay],
                                      [m for _, m, _ in lay], [int(p is not None) for _, _, p in lay])
        need = s["plan"].info()["workspace_bytes"]
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None


def _prepare_verify(case, g, s):
    lay = _verify_layout(case)
    rows, V = sum(len(p) for p in lay), case["vocab"]
    dtype = getattr(torch, case["dtype"])
    # the draft model's logits are the target's with noise: most drafts stay
    logits = _normal(g, rows, V, dtype=torch.float32).mul_(4.0)
    s["target"] = torch.softmax(logits, 1).to(dtype)
    logits.add_(_normal(g, rows, V, dtype=torch.float32).mul_(0.7))
    draft = torch.softmax(logits, 1).to(dtype)
    s["draft"] = None if case["kind"] == "best" else draft
    s["parents"] = _ints([x for p in lay for x in p])
    s["rows"], s["valid"] = _padded([len(p) for p in lay])
    first = [sum(len(p) for p in lay[:t]) for t in range(len(lay))]
    parent_row = _ints([f + max(x, 0) for f, p in zip(first, lay) for x in p], torch.int64)
    if case["kind"] == "best":  # the n-th child of a node holds its n-th best token
        order = [p[:i].count(x) for p in lay for i, x in enumerate(p)]
        best = torch.topk(draft.float(), min(V, max(order) + 1), dim=1).indices
        s["tokens"] = best[parent_row, _ints(order, torch.int64)].to(torch.int32)
    else:  # each child is drawn from its parent's row
        noise = torch.empty(rows, V, device=DEV).exponential_(generator=g)
        s["tokens"] = (draft.float()[parent_row] / noise).argmax(1).to(torch.int32)
        del noise
    s["u_accept"] = torch.rand(rows, generator=g, device=DEV)
    s["u_sample"] = torch.rand(len(lay), generator=g, device=DEV)
    n = max(len(p) for p in lay)
    s["path"] = torch.empty(len(lay), n, dtype=torch.int32, device=DEV)
    s["path_len"] = torch.empty(len(lay), dtype=torch.int32, device=DEV)
    s["next_token"] = torch.empty(len(lay), dtype=torch.int32, device=DEV)
    s["most_children"] = max(p.count(x) for p in lay for x in set(p))
    if own:
        import paper_2606_02964_amd as msa
        # the plan of the step whose rows these are: only its trees matter here
        m = [len(p) for p in lay]
        shape = msa.make_shape(len(lay), 8, 8, 128, -(-n // BS), sum(-(-x // BS) for x in m), 1.0)
        s["plan"] = msa.msa_plan_tree(shape, m, list(range(len(m) + 1)), [0] * len(m), m)
        s["workspace"] = torch.empty(msa.msa_tree_verify_workspace(s["plan"], V), dtype=torch.uint8, device=DEV)


def _prepare_weights(case, g, s):
    lay = _weights_layout(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    lens = [L for L, _ in lay]
    pos = [[p for a, n in segs for p in range(a, a + n)] for _, segs in lay]
    rows = sum(len(p) for p in pos)
    s["table"], s["k_cache"], _ = _cache(g, lens, hkv, d)
    s["q"] = _normal(g, rows, hq, d)
    s["scale"] = d ** -0.5
    s["rows"], s["valid"] = _padded([len(p) for p in pos])
    s["pos"] = _ints([x for p in pos for x in p], torch.int64)
    s["lse"] = torch.empty(rows, hq, device=DEV)
    x = _scores(s["q"], s["k_cache"], s["table"], s["rows"], s["scale"])
    x.masked_fill_(~_causal(s)[:, None, :, None, :], -math.inf)
    s["lse"][s["rows"][s["valid"]]] = torch.logsumexp(x, -1).permute(0, 2, 1, 3).reshape(*s["rows"].shape, hq)[s["valid"]]
    del x
    # what earlier steps have added up
    s["weights"] = torch.rand(len(lay), hkv, s["table"].shape[1] * BS, generator=g, device=DEV).mul_(4.0)
    if own:
        import paper_2606_02964_amd as msa
        shape = msa.make_shape(len(lay), hq, hkv, d, s["table"].shape[1], s["k_cache"].shape[0], s["scale"])
        indptr, segs = [0], [x for _, sg in lay for x in sg]
        for _, sg in lay:
            indptr.append(indptr[-1] + len(sg))
        s["plan"] = msa.msa_plan(shape, lens, indptr, [a for a, _ in segs], [n for _, n in segs])
        need = msa.msa_kv_weights_workspace(s["plan"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None


def _prepare_select(case, g, s):
    r = random.Random(case["layout_seed"])
    lens = _lengths(r, case["seqs"], case["ctx"])
    top = max(lens)
    # weights fall off with rank; sums of few steps, rounded coarsely, tie
    x = torch.rand(case["seqs"], case["lists"], top, generator=g, device=DEV).pow_(4.0).mul_(8.0)
    s["scores"] = (x * 32).round().div(32) if case["ties"] else x
    s["len"] = _ints(lens)
    keep = [min(L, int(L * case["part"]) + 8) for L in lens]
    s["keep"] = _ints(keep)
    s["first"], s["recent"] = 4, 16
    s["index"] = torch.full((case["seqs"], case["lists"], max(keep)), -1, dtype=torch.int32, device=DEV)
    s["count"] = torch.empty(case["seqs"], dtype=torch.int32, device=DEV)


def _prepare_compact(case, g, s):
    r = random.Random(case["layout_seed"])
    hkv, d = case["hkv"], case["d"]
    lens = _lengths(r, case["seqs"], case["ctx"])
    heads = 1 if case["shared"] else hkv
    if case["call"] == "commit":  # a path of a quarter of the slots, the root first
        n = max(1, case["slots"] // 4)
        total, base, counts = [L + case["slots"] for L in lens], lens, [n] * len(lens)
        among = [case["slots"]] * len(lens)
    else:
        total, base, counts = lens, [0] * len(lens), [min(L, int(L * case["part"]) + 1) for L in lens]
        among = lens
    s["table"], s["k_cache"], s["v_cache"] = _cache(g, total, hkv, d)
    order = torch.rand(len(lens), heads, max(among), generator=g, device=DEV)
    order.masked_fill_(torch.arange(max(among), device=DEV)[None, None, :] >= _ints(among)[:, None, None], 2.0)
    if case["call"] == "commit":
        order[:, :, 0] = -1.0
    # the first places of a random order, in ascending order, are kept
    rank = torch.argsort(torch.argsort(order, -1), -1)
    kept = rank < _ints(counts)[:, None, None]
    place = torch.cumsum(kept, -1) - 1
    index = torch.full((len(lens), heads, max(counts)), -1, dtype=torch.int32, device=DEV)
    b, h, j = torch.nonzero(kept, as_tuple=True)
    index[b, h, place[b, h, j]] = j.to(torch.int32)
    s["index"], s["base"], s["count"] = (index[:, 0] if case["shared"] else index), _ints(base), _ints(counts)
    if own:
        import paper_2606_02964_amd as msa
        s["shape"] = msa.make_shape(len(lens), hkv, hkv, d, s["table"].shape[1], s["k_cache"].shape[0], 1.0)


# ---- one pass ----

def run(s):
    return {"tree": _run_tree, "verify": _run_verify, "weights": _run_weights, "select": _run_select,
            "compact": _run_compact}[s["case"]["op"]](s)


def _keys(cache, table, is_v=False):
    """K or V in position order in 32 bits, [sequences, heads, positions, d]."""
    x = cache[table.clamp(min=0).long()].float()
    x = x.permute(0, 2, 1, 4, 3) if is_v else x.permute(0, 2, 1, 3, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _scores(q, k_cache, table, rows, scale):
    """Scaled scores [sequences, KV heads, rows, group, positions]."""
    k = _keys(k_cache, table)
    B, H, L, d = k.shape
    R, G = rows.shape[1], q.shape[1] // H
    x = q.float()[rows].reshape(B, R, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, R * G, d)
    return torch.matmul(x, k.transpose(2, 3)).mul_(scale).reshape(B, H, R, G, L)


def _causal(s):
    at = torch.arange(s["table"].shape[1] * BS, device=DEV)
    return (at[None, None, :] <= s["pos"][s["rows"]][:, :, None]) & s["valid"][:, :, None]


def _positions(s, pos):
    """Cache block and place in it of positions [sequences, n]."""
    return torch.gather(s["table"], 1, pos // BS).long(), pos % BS


def _related(parents, rows, valid):
    """Whether slot j is slot i or one of its ancestors, [trees, i, j]."""
    p = torch.where(valid, parents[rows], -1)
    at = torch.arange(rows.shape[1], device=DEV)
    rel = ((p[:, :, None] == at) | (at[:, None] == at)).float()
    for _ in range(max(1, rows.shape[1].bit_length())):  # twice the generations each time
        rel = (torch.matmul(rel, rel) > 0).float()
    return rel > 0


def _ancestors(s):
    """The mask words [tree rows, words] of the trees' parents."""
    rel = _related(s["parents"], s["tree_rows"], s["tree_valid"])
    words = s["mask"].shape[1]
    bits = torch.zeros(rel.shape[0], rel.shape[1], words * 64, dtype=torch.int64, device=DEV)
    bits[:, :, :rel.shape[2]] = rel.long()
    bits = bits.reshape(*bits.shape[:2], words, 64) << torch.arange(64, device=DEV)
    return bits.sum(-1)[s["tree_valid"]]


def _run_tree(s):
    call, out = s["case"]["call"], {}
    if own:
        import paper_2606_02964_amd as msa
        if call == "step":
            msa.msa_tree_mask(s["plan"], s["parents"], s["mask"])
        if call != "forward":
            msa.msa_kv_append(s["plan"], s["k_new"], s["v_new"], s["table"], s["k_cache"], s["v_cache"])
        msa.msa_tree_forward(s["plan"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["mask"], s["o"], s["lse"],
                             s["workspace"])
        out["o"], out["lse"] = s["o"], s["lse"]
    else:
        if call == "step":
            s["mask"].copy_(_ancestors(s))
        place = torch.arange(s["rows"].shape[1], device=DEV)
        pos = s["start"][:, None] + place[None, :]  # [sequences, rows]
        if call != "forward":
            blk, at = _positions(s, torch.where(s["valid"], pos, 0))
            blk, at, rows = blk[s["valid"]], at[s["valid"]], s["rows"][s["valid"]]
            s["k_cache"][blk, :, at] = s["k_new"][rows]
            s["v_cache"][blk, :, :, at] = s["v_new"][rows]
        x = _scores(s["q"], s["k_cache"], s["table"], s["rows"], s["scale"])
        at = torch.arange(x.shape[-1], device=DEV)
        # a tree's row sees the context and the slots of its mask, a causal one every position up to its own
        rel = at[None, :] - s["start"][:, None]
        bit = rel.clamp(0, s["mask"].shape[1] * 64 - 1)[:, None, :].expand(-1, len(place), -1)
        mask_row = torch.where(s["valid"], s["mask_row"][s["rows"]], -1)
        words = s["mask"][mask_row.clamp(min=0)]
        seen = (torch.gather(words, 2, bit // 64) >> (bit % 64)) & 1
        seen = (seen > 0) | (rel < 0)[:, None, :] | (mask_row < 0)[:, :, None]
        seen &= (at[None, None, :] <= pos[:, :, None]) & s["valid"][:, :, None]
        x.masked_fill_(~seen[:, None, :, None, :], -math.inf)
        m = x.amax(-1, keepdim=True).clamp(min=-3e38)
        x.sub_(m).exp_()
        l = x.sum(-1, keepdim=True)
        B, H, R, G, L = x.shape
        o = torch.matmul(x.reshape(B, H, R * G, L), _keys(s["v_cache"], s["table"], True)).reshape(B, H, R, G, -1)
        o = torch.where(l > 0, o / l, 0.0).permute(0, 2, 1, 3, 4).reshape(B, R, H * G, -1)
        s["o"][s["rows"][s["valid"]]] = o[s["valid"]].to(torch.bfloat16)
        if s["lse"] is not None:
            lse = (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, R, H * G)
            s["lse"][s["rows"][s["valid"]]] = lse[s["valid"]]
        out["o"], out["lse"] = s["o"], s["lse"]
    if call == "step":
        out["mask"] = s["mask"]
    if call != "forward":
        out["k_cache"], out["v_cache"] = s["k_cache"], s["v_cache"]
    return out


def _run_verify(s):
    if own:
        import paper_2606_02964_amd as msa
        msa.msa_tree_verify(s["plan"], s["target"], s["tokens"], s["parents"], s["u_accept"], s["u_sample"], s["path"],
                            s["path_len"], s["next_token"], s["draft"], s["workspace"])
        return {"path": s["path"], "path_len": s["path_len"], "next_token": s["next_token"]}
    # in 64 bits: sums over the vocabulary decide between neighbouring tokens
    T, S = s["rows"].shape
    at = torch.arange(S, device=DEV)
    parent = torch.where(s["valid"], s["parents"][s["rows"]], -1).long()
    token = s["tokens"][s["rows"]].long()
    parent_row = torch.gather(s["rows"], 1, parent.clamp(min=0))
    p = s["target"][parent_row, token].double()
    u = s["u_accept"][s["rows"]].double()
    sibling = (parent[:, :, None] == parent[:, None, :]) & (at[None, :] < at[:, None]) & (parent >= 0)[:, :, None]
    # the residual of a node after its first n children failed is max(a p - b q, 0)
    # with mass P (drawn drafts), or p without those children's tokens (best drafts)
    if s["draft"] is None:
        twice = (sibling & (token[:, :, None] == token[:, None, :])).any(-1)
        p = torch.where(twice, 0.0, p)
        mass = 1.0 - torch.where(sibling, p[:, None, :], 0.0).sum(-1)
        passed = u * mass < p
    else:
        q = s["draft"][parent_row, token].double()
        rank = sibling.sum(-1)
        a, b = torch.ones(T, S, device=DEV, dtype=torch.float64), torch.ones(T, S, device=DEV, dtype=torch.float64)
        scale, less = [a], [b]  # by node, after one failed child, after two, ...
        passed = (rank == 0) & (u * q < p)
        P_rows, Q_rows = s["target"].double()[s["rows"]], s["draft"].double()[s["rows"]]
        for n in range(1, s["most_children"]):
            mass = (a[:, :, None] * P_rows - b[:, :, None] * Q_rows).clamp_(min=0).sum(-1)
            ap, bp = torch.gather(a, 1, parent.clamp(min=0)), torch.gather(b, 1, parent.clamp(min=0))
            mp = torch.gather(mass, 1, parent.clamp(min=0))
            passed |= (rank == n) & (u * q * mp < (ap * p - bp * q).clamp(min=0))
            a, b = a / mass, b / mass + 1.0
            scale.append(a)
            less.append(b)
    passed &= (parent >= 0) & s["valid"]
    taken = passed & ~(sibling & passed[:, None, :]).any(-1)
    taken |= at[None, :] == 0
    on_path = ~(_related(s["parents"], s["rows"], s["valid"]) & ~taken[:, None, :]).any(-1) & s["valid"]
    s["path_len"].copy_(on_path.sum(1))
    s["path"].copy_(torch.where(on_path, at, S).sort(1).values)
    s["path"].masked_fill_(s["path"] == S, -1)
    # the next token: drawn from what the last node's failed children left
    last = torch.where(on_path, at, 0).amax(1)
    row = torch.gather(s["rows"], 1, last[:, None])[:, 0]
    w, failed = s["target"][row].double(), (parent == last[:, None]) & s["valid"]
    if s["draft"] is None:
        rest = w.clone()
        t, j = torch.nonzero(failed, as_tuple=True)
        rest[t, token[t, j]] = 0.0
    else:
        n = failed.sum(1)
        which = ((n - 1).clamp(min=0), torch.arange(T, device=DEV), last)
        rest = torch.stack(scale)[which][:, None] * w - torch.stack(less)[which][:, None] * s["draft"][row].double()
        rest = torch.where((n > 0)[:, None], rest.clamp(min=0), w)
    total = torch.cumsum(rest, 1)
    total = torch.where(total[:, -1:] > 0, total, torch.cumsum(w, 1))
    s["next_token"].copy_((total <= s["u_sample"].double()[:, None] * total[:, -1:]).sum(1))
    return {"path": s["path"], "path_len": s["path_len"], "next_token": s["next_token"]}


def _run_weights(s):
    if own:
        import paper_2606_02964_amd as msa
        msa.msa_kv_weights(s["plan"], s["q"], s["k_cache"], s["table"], s["lse"], s["weights"], s["workspace"])
        return s["weights"]
    x = _scores(s["q"], s["k_cache"], s["table"], s["rows"], s["scale"])
    B, H, R, G, L = x.shape
    x.sub_(s["lse"][s["rows"]].reshape(B, R, H, G).permute(0, 2, 1, 3)[..., None]).exp_()
    x.masked_fill_(~_causal(s)[:, None, :, None, :], 0.0)
    s["weights"].add_(x.sum((2, 3)))
    return s["weights"]


def _run_select(s):
    if own:
        import paper_2606_02964_amd as msa
        msa.msa_kv_select(s["scores"], s["len"], s["keep"], s["index"], s["count"], s["first"], s["recent"])
        return {"index": s["index"], "count": s["count"]}
    n, at = s["len"][:, None, None], torch.arange(s["scores"].shape[2], device=DEV)
    keep = torch.minimum(s["keep"], s["len"])[:, None, None]
    recent = torch.clamp(keep, max=s["recent"])
    first = torch.clamp(keep - recent, max=s["first"])
    x = torch.where((at < first) | (at >= n - recent), math.inf, s["scores"])
    x = torch.where(at < n, x, -math.inf)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices  # equal scores: the lower position first
    order = torch.where(at < keep, order, s["scores"].shape[2]).sort(-1).values[:, :, :s["index"].shape[2]]
    s["index"].copy_(torch.where(at[:s["index"].shape[2]] < keep, order, -1))
    s["count"].copy_(keep[:, 0, 0])
    return {"index": s["index"], "count": s["count"]}


def _run_compact(s):
    if own:
        import paper_2606_02964_amd as msa
        msa.msa_kv_compact(s["shape"], s["base"], s["index"], s["count"], s["table"], s["k_cache"], s["v_cache"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    index = s["index"] if s["index"].dim() == 3 else s["index"][:, None]
    H = s["k_cache"].shape[1]
    index = index.expand(-1, H, -1).long()
    place = torch.arange(index.shape[2], device=DEV)
    b, h, i = torch.nonzero((place[None, None, :] < s["count"][:, None, None]).expand_as(index), as_tuple=True)
    src, dst = s["base"].long()[b] + index[b, h, i], s["base"].long()[b] + i
    from_blk, to_blk = s["table"][b, src // BS].long(), s["table"][b, dst // BS].long()
    k, v = s["k_cache"][from_blk, h, src % BS], s["v_cache"][from_blk, h, :, src % BS]
    s["k_cache"][to_blk, h, dst % BS] = k
    s["v_cache"][to_blk, h, :, dst % BS] = v
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


# ---- the same in 64 bits, sequence by sequence ----

def _rows64(cache, table, L, head, is_v):
    blocks = cache[table[:-(-L // BS)].long(), head]
    blocks = blocks.transpose(1, 2) if is_v else blocks
    return blocks.reshape(-1, blocks.shape[-1])[:L].double()


def exact(case, seed):
    if case["op"] in ("verify", "select"):
        return None  # whole numbers
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    return {"tree": _exact_tree, "weights": _exact_weights, "compact": _exact_compact}[case["op"]](case, s)


def _exact_tree(case, s):
    lay, out = _tree_layout(case), {}
    if case["call"] != "forward":
        row = 0
        for b, (c, m, _) in enumerate(lay):
            for i in range(m):
                blk, at = int(s["table"][b, (c + i) // BS]), (c + i) % BS
                s["k_cache"][blk, :, at], s["v_cache"][blk, :, :, at] = s["k_new"][row + i], s["v_new"][row + i]
            row += m
        out["k_cache"], out["v_cache"] = s["k_cache"], s["v_cache"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    G = hq // hkv
    out["o"] = torch.zeros(len(s["q"]), hq, d, dtype=torch.float64, device=DEV)
    out["lse"] = torch.full((len(s["q"]), hq), -math.inf, dtype=torch.float64, device=DEV)
    row = 0
    for b, (c, m, parents) in enumerate(lay):
        seen = torch.ones(m, m, dtype=torch.bool).tril()
        if parents is not None:
            seen = torch.zeros(m, m, dtype=torch.bool)
            for i, x in enumerate(parents):
                if x >= 0:
                    seen[i] = seen[x]
                seen[i, i] = True
        seen = seen.to(DEV).repeat_interleave(G, 0)
        for h in range(hkv):
            k, v = (_rows64(s[n], s["table"][b], c + m, h, n == "v_cache") for n in ("k_cache", "v_cache"))
            q = s["q"][row:row + m, h * G:(h + 1) * G].double().reshape(m * G, d)
            x = (q @ k.T) * d ** -0.5
            x[:, c:].masked_fill_(~seen, -math.inf)
            l = torch.logsumexp(x, 1)
            out["o"][row:row + m, h * G:(h + 1) * G] = (torch.exp(x - l[:, None]) @ v).view(m, G, d)
            out["lse"][row:row + m, h * G:(h + 1) * G] = l.view(m, G)
        row += m
    if s["lse"] is None:
        out["lse"] = None
    if case["call"] == "step":
        out["mask"] = None
    return out


def _exact_weights(case, s):
    out = s["weights"].double()
    G, row = case["hq"] // case["hkv"], 0
    for b, (L, segs) in enumerate(_weights_layout(case)):
        for a, n in segs:
            for h in range(case["hkv"]):
                k = _rows64(s["k_cache"], s["table"][b], a + n, h, False)
                for i in range(0, n, 1024):
                    m = min(1024, n - i)
                    q = s["q"][row + i:row + i + m, h * G:(h + 1) * G].double().reshape(m * G, -1)
                    x = (q @ k.T) * case["d"] ** -0.5
                    x = torch.exp(x - s["lse"][row + i:row + i + m, h * G:(h + 1) * G].double().reshape(-1, 1))
                    at = torch.arange(a + i, a + i + m, device=DEV).repeat_interleave(G)
                    x *= torch.arange(a + n, device=DEV)[None, :] <= at[:, None]
                    out[b, h, :a + n] += x.sum(0)
            row += n
    return out


def _exact_compact(case, s):
    out = {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
    for b in range(case["seqs"]):
        n, base = int(s["count"][b]), int(s["base"][b])
        dst = torch.arange(base, base + n, device=DEV)
        to = s["table"][b][dst // BS].long()
        for h in range(case["hkv"]):
            src = base + (s["index"][b] if case["shared"] else s["index"][b, h])[:n].long()
            at = s["table"][b][src // BS].long()
            out["k_cache"][to, h, dst % BS] = s["k_cache"][at, h, src % BS].double()
            out["v_cache"][to, h, :, dst % BS] = s["v_cache"][at, h, :, src % BS].double()
    return out
