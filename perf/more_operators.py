"""The measured calls of rotary positions, the 8-bit cache and windowed attention.

A case is one pass as a layer of a serving step makes it, with the plan, the
workspace and the buffers that such a program keeps from step to step:

* ``rope``: q and the new keys rotated by their positions, K and V written into
  the paged cache;
* ``write``: new K and V written into an 8-bit cache (e4m3 values, a power of two
  for each token and KV head), and the sequences read back into a bf16 cache;
* ``attn``: attention over the paged cache, where ``cache`` is "fp8" or a
  ``window`` is set (keys of the latest ``window`` positions and the first
  ``sinks``), alone ("forward") or after the rotation and the write of the new
  tokens ("layer").

Sizes are generic: the head layouts of this repository's workloads, contexts
from tens of tokens to 64K, one new token to whole prompts.  A case's layout
depends on its fields only, its values and the placement of its cache blocks on
the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
BS = 16  # tokens of a cache block
E4M3 = torch.float8_e4m3fn
E_MIN, E_BIAS, E4M3_MAX = -110, 127, 448.0

# (query heads, KV heads, head_dim): an 8B and a 70B layer, one tensor-parallel
# rank of each, and heads without grouping at the smaller head dimension
HEADS = ((32, 8, 128), (64, 8, 128), (8, 2, 128), (16, 2, 128), (16, 16, 64), (4, 4, 64))
MOST = {"rope": 16384 * 48 * 128, "write": 32 * 8 * 128 * 8192, "attn": 12000 * 32 * 12000}


def listed():
    def rope(name, layout, seqs, ctx, new, heads=(32, 8, 128), rot=0, pairs="half", far=0):
        return dict(name=name, op="rope", layout=layout, seqs=seqs, ctx=ctx, new=new, hq=heads[0], hkv=heads[1], d=heads[2],
                    rot=rot or heads[2], pairs=pairs, far=far, layout_seed=3)

    def write(name, layout, seqs, ctx, new, heads=(32, 8, 128)):
        return dict(name=name, op="write", layout=layout, seqs=seqs, ctx=ctx, new=new, hkv=heads[1], d=heads[2], layout_seed=3)

    def attn(name, cache, layout, seqs, ctx, new, window=0, sinks=0, heads=(32, 8, 128), call="forward", lse=False):
        return dict(name=name, op="attn", cache=cache, layout=layout, seqs=seqs, ctx=ctx, new=new, window=window, sinks=sinks,
                    hq=heads[0], hkv=heads[1], d=heads[2], call=call, rot=heads[2], pairs="half", far=0, lse=lse, layout_seed=3)

    return [
        # one user's next token: the smallest call
        rope("rope_one", "end", 1, 4000, 1, heads=(8, 2, 128)),
        # a chunk of a prompt for each of a batch, and a piece recomputed earlier on
        rope("rope_chunks", "pieces", 8, 8192, 1024),
        # a quarter of each head rotated in neighbouring pairs, positions far past the places in the cache
        rope("rope_part", "end", 40, 3001, 100, heads=(16, 16, 64), rot=16, pairs="interleaved", far=900000),
        # a batch's chunks into the 8-bit cache, whose sequences then go back to bf16
        write("write_chunks", "end", 16, 8000, 512),
        # one token for each of a large batch, short sequences
        write("write_tokens", "end", 200, 300, 1, heads=(8, 2, 128)),
        # a decoding batch over the 8-bit cache
        attn("fp8_decode", "fp8", "end", 64, 8000, 1, lse=True),
        # one user's token: rotation, write and attention over a long context
        attn("fp8_one", "fp8", "end", 1, 30001, 1, call="layer"),
        # chunks of prompts over the 8-bit cache, at the end and recomputed earlier on
        attn("fp8_chunks", "fp8", "pieces", 8, 8192, 512),
        # one user's next token with a window: the smallest attention
        attn("window_one", "bf16", "end", 1, 700, 1, window=256, sinks=4, heads=(4, 4, 64), call="layer"),
        # a decoding batch with long contexts, of which a window is seen
        attn("window_decode", "bf16", "end", 48, 32768, 1, window=4096, sinks=4),
        # a whole prompt: the largest call
        attn("window_prompt", "bf16", "prompt", 1, 12000, 0, window=1024, sinks=64, lse=True),
        # the same with the 8-bit cache, for a batch of shorter prompts' last chunks
        attn("window_fp8", "fp8", "end", 12, 10001, 300, window=2000, sinks=20, heads=(64, 8, 128)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any operator, sizes spread over their logarithm, odd
    ones among them, no larger than the largest listed case."""
    while True:
        op = rng.choice(("rope", "write", "attn", "attn"))
        hq, hkv, d = rng.choice(HEADS)
        layout = rng.choice(("end", "end", "pieces", "prompt"))
        case = dict(op=op, layout_seed=rng.randrange(1 << 20), layout=layout, hkv=hkv, d=d,
                    seqs=_log_int(rng, 1, 8 if layout == "prompt" else 64),
                    ctx=_log_int(rng, 16, 12000 if layout == "prompt" else 40000),
                    new=0 if layout == "prompt" else rng.choice((1, _log_int(rng, 2, 1024))))
        rows = case["seqs"] * {"end": case["new"], "pieces": 2 * case["new"], "prompt": case["ctx"]}[layout]
        turn = dict(rot=rng.choice((d, d, d // 2, d // 4)), pairs=rng.choice(("half", "interleaved")),
                    far=rng.choice((0, 0, _log_int(rng, 1000, 1000000))))
        if op == "rope":
            case.update(hq=hq, **turn)
            cost = rows * (hq + 2 * hkv) * d
        elif op == "write":
            cost = case["seqs"] * hkv * d * case["ctx"]
        else:
            cache = rng.choice(("fp8", "bf16"))
            windowed = cache == "bf16" or rng.random() < 0.3
            case.update(cache=cache, hq=hq, window=_log_int(rng, 1, 8192) if windowed else 0,
                        sinks=rng.choice((0, 4, _log_int(rng, 1, 200))) if windowed else 0,
                        call=rng.choice(("forward", "forward", "layer")), lse=rng.random() < 0.5, **turn)
            case["lse"] &= case["call"] == "forward"  # (a rotated key next to a rounding border moves the lse of few keys by more than 32 bits)
            cost = max(rows * hq * case["ctx"], 2 * case["seqs"] * hkv * d * case["ctx"])
        if cost <= MOST[op]:
            return case


# ---- layouts: plain host numbers from a case's fields ----

def _layout(case):
    """Context length and (start, length) query segments of each sequence."""
    r = random.Random(case["layout_seed"])
    out = []
    for _ in range(case["seqs"]):
        L = case["ctx"] if case["seqs"] == 1 else r.randint(max(1, case["ctx"] // 4), case["ctx"])
        n = L if case["layout"] == "prompt" else min(L, case["new"] if case["new"] <= 1 else r.randint((case["new"] + 1) // 2, case["new"]))
        segs = [(L - n, n)]
        if case["layout"] == "pieces" and (L - n) // 2 > 0:
            m = min(n, (L - n) // 2)
            segs.insert(0, ((L - n - m) // 2, m))
        out.append((L, segs))
    return out


def _seen(case, p):
    """Keys that the row at position p sees."""
    if not case["window"] or p < case["window"]:
        return p + 1
    return case["window"] + min(case["sinks"], p - case["window"] + 1)


def _seen_by_any(case, segs):
    """Keys that some row of the segments sees."""
    at = set()
    end = 0
    for a, n in segs:
        lo = max(0, a - case["window"] + 1) if case["window"] else 0
        lo = max(lo, end)
        at.add((lo, max(lo, a + n)))
        end = max(end, a + n)
    total = sum(b - a for a, b in at)
    first = min(a for a, b in at)
    return total + min(case["sinks"], first)


def work(case):
    lay = _layout(case)
    rows = sum(n for _, segs in lay for _, n in segs)
    if case["op"] == "rope":
        return {"bytes": rows * (case["hq"] + 2 * case["hkv"]) * case["d"] * 4, "flops": rows * (case["hq"] + case["hkv"]) * case["rot"] * 3}
    if case["op"] == "write":
        # the new numbers read, and written in 8 bits; all read in 8 bits and written in 16
        back = sum(L for L, _ in lay) * case["hkv"] * 2
        return {"bytes": rows * case["hkv"] * 2 * (3 * case["d"] + 1) + back * (3 * case["d"] + 1), "flops": back * case["d"]}
    key = 2 * case["d"] + 2 if case["cache"] == "fp8" else 4 * case["d"]
    nbytes = 4 * rows * case["hq"] * case["d"] + (4 * rows * case["hq"] if case["lse"] else 0)
    nbytes += sum(_seen_by_any(case, segs) for _, segs in lay) * case["hkv"] * key
    if case["call"] == "layer":  # q rotated in place, new keys and values read and written
        nbytes += 4 * rows * case["hq"] * case["d"] + rows * case["hkv"] * (4 * case["d"] + key)
    pairs = sum(_seen(case, p) for _, segs in lay for a, n in segs for p in range(a, a + n))
    return {"bytes": nbytes, "flops": 4 * case["d"] * case["hq"] * pairs}


# ---- inputs ----

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _ints(values, dtype=torch.int32):
    return torch.tensor(values, dtype=dtype, device=DEV)


def _table(g, lens):
    """Scattered cache blocks for sequences of these lengths, and their number."""
    counts = [-(-L // BS) for L in lens]
    n, most = sum(counts), max(counts)
    table = torch.full((len(lens), most), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(most, device=DEV)[None, :] < _ints(counts)[:, None]] = \
        torch.randperm(n, generator=g, device=DEV).to(torch.int32)
    return table, n


def _two(e):
    """2^e in 32 bits, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _exponent(x):
    """The power of two for each row of numbers: the smallest e with max|x| <= 448 * 2^e, from E_MIN on."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    return torch.where(m > 0, e - 9 + (m > 0.875), E_MIN).clamp(min=E_MIN)


def _quantised(x):
    """e4m3 bytes of x [..., d] and the byte of its power of two [...]."""
    e = _exponent(x)
    return (x * _two(-e)).to(E4M3).view(torch.uint8), (e + E_BIAS).to(torch.uint8).squeeze(-1)


def _cache8(g, n, hkv, d):
    """A quantised cache of n blocks: values K [n, hkv, BS, d], V [n, hkv, d, BS], powers of two [n, hkv, BS] each."""
    # keys differ in size from channel to channel and token to token, as a model's do
    k = _normal(g, n, hkv, BS, d).float() * torch.rand(d, generator=g, device=DEV).mul_(1.5).add_(0.25)
    v = _normal(g, n, hkv, BS, d).float() * torch.rand(n, hkv, BS, 1, generator=g, device=DEV).mul_(1.5).add_(0.25)
    k, ks = _quantised(k)
    v, vs = _quantised(v)
    return k, v.transpose(2, 3).contiguous(), ks, vs


def prepare(case, seed):
    g, s = _generator(seed), {"case": case}
    lay = _layout(case)
    hq, hkv, d = case.get("hq", case["hkv"]), case["hkv"], case["d"]
    lens = [L for L, _ in lay]
    pos = [[p for a, n in segs for p in range(a, a + n)] for _, segs in lay]
    counts = [len(p) for p in pos]
    rows = sum(counts)
    fp8 = case["op"] == "write" or case.get("cache") == "fp8"
    s["table"], n = _table(g, lens)
    if fp8:
        s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"] = _cache8(g, n, hkv, d)
    else:
        s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"] = _normal(g, n, hkv, BS, d), _normal(g, n, hkv, d, BS), None, None
    qkv = _normal(g, rows, hq + 2 * hkv, d)  # one fused projection's output, as a model has it
    s["q"], s["k_new"], s["v_new"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    # where each row stands: its sequence, its place in it, and the rows of each sequence side by side
    s["pos"] = _ints([x for p in pos for x in p], torch.int64)
    s["seq"] = _ints([b for b, c in enumerate(counts) for _ in range(c)], torch.int64)
    start = torch.cumsum(_ints([0] + counts, torch.int64), 0)
    place = torch.arange(max(counts), device=DEV)
    s["valid"] = place[None, :] < _ints(counts)[:, None]
    s["rows"] = torch.where(s["valid"], start[:-1, None] + place[None, :], 0)
    s["scale"] = d ** -0.5
    if "rot" in case:
        # frequencies stretched for long contexts: the slow ones by 8, the fast ones not at all
        i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
        f = 500000.0 ** (-2.0 * i / case["rot"])
        keep = ((8192.0 * f / (2 * math.pi) - 1.0) / 3.0).clamp(0.0, 1.0)
        s["freq"] = f * keep + f / 8.0 * (1.0 - keep)
        s["angle_pos"] = (s["pos"] + case["far"]).to(torch.int32) if case["far"] else None
        s["q_out"] = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEV)
    if case["op"] == "write":  # the bf16 cache that the sequences are read back into
        s["end"] = _ints(lens)
        s["to_table"], _ = _table(g, lens)
        s["k_back"] = torch.zeros(n, hkv, BS, d, dtype=torch.bfloat16, device=DEV)
        s["v_back"] = torch.zeros(n, hkv, d, BS, dtype=torch.bfloat16, device=DEV)
    if case["op"] == "attn":
        s["o"] = torch.empty(rows, hq, d, dtype=torch.bfloat16, device=DEV)
        s["lse"] = torch.empty(rows, hq, dtype=torch.float32, device=DEV) if case["lse"] else None
        if case["call"] == "forward":
            s["q_out"] = s["q"].contiguous()
    if own:
        import paper_2606_02964_amd as msa
        shape = msa.make_shape(len(lay), hq, hkv, d, s["table"].shape[1], n, s["scale"])
        indptr, segs = [0], [x for _, sg in lay for x in sg]
        for _, sg in lay:
            indptr.append(indptr[-1] + len(sg))
        host = (shape, lens, indptr, [a for a, _ in segs], [m for _, m in segs])
        s["plan"] = msa.msa_plan_window(*host, case["window"], case["sinks"]) if case.get("window") else msa.msa_plan(*host)
        s["shape"] = shape
        need = s["plan"].info()["workspace_bytes"]
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
        if "rot" in case:
            s["rope"] = msa.make_rope(s["freq"], msa.MSA_ROPE_HALF if case["pairs"] == "half" else msa.MSA_ROPE_INTERLEAVED)
    return s


# ---- one pass ----

def run(s):
    return {"rope": _run_rope, "write": _run_write, "attn": _run_attn}[s["case"]["op"]](s)


def _rotated(s, x):
    """x [rows, heads, d] in 32 bits, rotated by its positions."""
    p = s["pos"] if s["angle_pos"] is None else s["angle_pos"]
    t = p.double()[:, None, None] * s["freq"]
    c, w = torch.cos(t).float(), torch.sin(t).float()
    y = x.float().clone()
    R = s["case"]["rot"]
    a, b = (slice(0, R // 2), slice(R // 2, R)) if s["case"]["pairs"] == "half" else (slice(0, R, 2), slice(1, R, 2))
    x0, x1 = x[..., a].float(), x[..., b].float()
    y[..., a] = x0 * c - x1 * w
    y[..., b] = x1 * c + x0 * w
    return y


def _store(s, k, v):
    """K and V [rows, heads, d] in 32 bits into the cache, at the rows' places."""
    blk, at = s["table"][s["seq"], s["pos"] // BS].long(), s["pos"] % BS
    if s["k_scale"] is None:
        s["k_cache"][blk, :, at] = k.to(torch.bfloat16)
        s["v_cache"][blk, :, :, at] = v.to(torch.bfloat16)
    else:
        s["k_cache"][blk, :, at], s["k_scale"][blk, :, at] = _quantised(k)
        s["v_cache"][blk, :, :, at], s["v_scale"][blk, :, at] = _quantised(v)


def _turn_and_store(s):
    s["q_out"].copy_(_rotated(s, s["q"]))
    _store(s, _rotated(s, s["k_new"]), s["v_new"].float())


def _values(s):
    """The cache's K [blocks, heads, BS, d] and V [blocks, heads, d, BS] in 32 bits."""
    if s["k_scale"] is None:
        return s["k_cache"].float(), s["v_cache"].float()
    ks, vs = _two(s["k_scale"].int() - E_BIAS), _two(s["v_scale"].int() - E_BIAS)
    return s["k_cache"].view(E4M3).float() * ks[:, :, :, None], s["v_cache"].view(E4M3).float() * vs[:, :, None, :]


def _own_rope(s):
    import paper_2606_02964_amd as msa
    msa.msa_rope_append(s["plan"], s["rope"], s["q"], s["q_out"], s["k_new"], s["v_new"], s["table"], s["k_cache"],
                        s["v_cache"], s["k_scale"], s["v_scale"], s["angle_pos"])


def _run_rope(s):
    if own:
        _own_rope(s)
    else:
        _turn_and_store(s)
    return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _run_write(s):
    out = {"k": s["k_back"], "v": s["v_back"]}
    if own:
        import paper_2606_02964_amd as msa
        msa.msa_fp8_append(s["plan"], s["k_new"], s["v_new"], s["table"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"])
        msa.msa_fp8_read(s["shape"], None, s["end"], s["case"]["ctx"], s["table"], s["k_cache"], s["v_cache"], s["k_scale"],
                         s["v_scale"], s["shape"], s["to_table"], s["k_back"], s["v_back"])
        return out
    _store(s, s["k_new"].float(), s["v_new"].float())
    k, v = _values(s)
    at = torch.arange(s["table"].shape[1] * BS, device=DEV)
    b, p = torch.nonzero(at[None, :] < s["end"][:, None], as_tuple=True)
    blk, to = s["table"][b, p // BS].long(), s["to_table"][b, p // BS].long()
    s["k_back"][to, :, p % BS] = k[blk, :, p % BS].to(torch.bfloat16)
    s["v_back"][to, :, :, p % BS] = v[blk, :, :, p % BS].to(torch.bfloat16)
    return out


def _run_attn(s):
    case = s["case"]
    if own:
        import paper_2606_02964_amd as msa
        if case["call"] == "layer":
            _own_rope(s)
        if case["cache"] == "fp8":
            msa.msa_fp8_forward(s["plan"], s["q_out"], s["k_cache"], s["v_cache"], s["k_scale"], s["v_scale"], s["table"],
                                s["o"], s["lse"], s["workspace"])
        else:
            msa.msa_forward(s["plan"], s["q_out"], s["k_cache"], s["v_cache"], s["table"], s["o"], s["lse"], s["workspace"])
        return {"o": s["o"], "lse": s["lse"]}
    if case["call"] == "layer":
        _turn_and_store(s)
    k, v = _values(s)
    table = s["table"].clamp(min=0).long()
    k = k[table].permute(0, 2, 1, 3, 4).flatten(2, 3)  # [sequences, KV heads, positions, d]
    v = v[table].permute(0, 2, 1, 4, 3).flatten(2, 3)
    B, H, L, d = k.shape
    R, G = s["rows"].shape[1], case["hq"] // H
    x = s["q_out"].float()[s["rows"]].reshape(B, R, H, G, d).permute(0, 2, 1, 3, 4).reshape(B, H, R * G, d)
    x = torch.matmul(x, k.transpose(2, 3)).mul_(s["scale"]).reshape(B, H, R, G, L)
    at, p = torch.arange(L, device=DEV), s["pos"][s["rows"]][:, :, None]
    seen = at <= p
    if case["window"]:
        seen &= (at > p - case["window"]) | (at < case["sinks"])
    x.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    m = x.amax(-1, keepdim=True)
    x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(B, H, R * G, L), v).reshape(B, H, R, G, d)
    o = (o / l).permute(0, 2, 1, 3, 4).reshape(B, R, H * G, d)
    s["o"][s["rows"][s["valid"]]] = o[s["valid"]].to(torch.bfloat16)
    if s["lse"] is not None:
        lse = (m + l.log()).squeeze(-1).permute(0, 2, 1, 3).reshape(B, R, H * G)
        s["lse"][s["rows"][s["valid"]]] = lse[s["valid"]]
    return {"o": s["o"], "lse": s["lse"]}


# ---- the same in 64 bits, by the definitions ----

def _exact_turn(case, s, x):
    """Pairs of channels as complex numbers, turned by the angle."""
    p = (s["pos"] + case["far"]).double()
    turn = torch.polar(torch.ones_like(p[:, None] * s["freq"]), p[:, None] * s["freq"])[:, None, :]
    x, R = x.double(), case["rot"]
    if case["pairs"] == "half":
        z = torch.complex(x[..., :R // 2], x[..., R // 2:R]) * turn
        y = torch.cat((z.real, z.imag), -1)
    else:
        z = torch.complex(x[..., 0:R:2], x[..., 1:R:2]) * turn
        y = torch.stack((z.real, z.imag), -1).flatten(-2)
    return torch.cat((y, x[..., R:]), -1)


def _exact_two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_round8(x):
    """x [..., d] as its row's 8-bit numbers stand for it."""
    top = (x.abs().amax(-1, keepdim=True) / 448.0).clamp(min=2.0 ** E_MIN)
    half, e = torch.frexp(top)  # top = half * 2^e, 0.5 <= half < 1
    step = _exact_two(torch.where(half == 0.5, e - 1, e))
    y = x / step
    # three bits behind the leading one, from 2^-6 on; multiples of 2^-9 below
    ulp = _exact_two(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / ulp) * ulp * step


def exact(case, seed):
    global own
    was, own = own, False
    s = prepare(case, seed)
    own = was
    layer = case["op"] != "attn" or case["call"] == "layer"
    fp8 = s["k_scale"] is not None
    # K and V of each block in 64 bits, [blocks, heads, BS, d]
    k, v = s["k_cache"], s["v_cache"].transpose(2, 3)
    if fp8:
        k = k.view(E4M3).double() * _exact_two(s["k_scale"].int() - E_BIAS)[..., None]
        v = v.contiguous().view(E4M3).double() * _exact_two(s["v_scale"].int() - E_BIAS)[..., None]
    else:
        k, v = k.double(), v.double()
    q = s["q"].double() if layer else s["q_out"].double()
    if layer:
        k_new, v_new = s["k_new"].double(), s["v_new"].double()
        if case["op"] != "write":
            q, k_new = _exact_turn(case, s, s["q"]), _exact_turn(case, s, s["k_new"])
        if fp8:
            k_new, v_new = _exact_round8(k_new), _exact_round8(v_new)
        elif case["op"] == "attn":  # the cache holds 16 bits
            q, k_new = q.to(torch.bfloat16).double(), k_new.to(torch.bfloat16).double()
        if fp8 and case["op"] == "attn":
            q = q.to(torch.bfloat16).double()
        blk = s["table"].long()[s["seq"], s["pos"] // BS]
        k[blk, :, s["pos"] % BS], v[blk, :, s["pos"] % BS] = k_new, v_new
    if case["op"] == "rope":
        return {"q": q, "k_cache": k, "v_cache": v.transpose(2, 3)}
    lay = _layout(case)
    if case["op"] == "write":
        k_back, v_back = torch.zeros_like(k), torch.zeros_like(v)
        for b, (L, _) in enumerate(lay):
            p = torch.arange(L, device=DEV)
            src, dst = s["table"][b].long()[p // BS], s["to_table"][b].long()[p // BS]
            k_back[dst, :, p % BS], v_back[dst, :, p % BS] = k[src, :, p % BS], v[src, :, p % BS]
        return {"k": k_back, "v": v_back.transpose(2, 3)}
    out = {"o": torch.zeros(q.shape, dtype=torch.float64, device=DEV),
           "lse": torch.zeros(q.shape[:2], dtype=torch.float64, device=DEV)}
    G, row = case["hq"] // case["hkv"], 0
    for b, (L, segs) in enumerate(lay):
        blocks = s["table"][b, :-(-L // BS)].long()
        for a, n in segs:
            for i in range(0, n, 1024):
                m = min(1024, n - i)
                p = torch.arange(a + i, a + i + m, device=DEV).repeat_interleave(G)[:, None]
                j = torch.arange(a + i + m, device=DEV)[None, :]
                hidden = j > p
                if case["window"]:
                    hidden |= (p - j >= case["window"]) & (j >= case["sinks"])
                for h in range(case["hkv"]):
                    kh, vh = k[blocks, h].flatten(0, 1)[:a + i + m], v[blocks, h].flatten(0, 1)[:a + i + m]
                    x = q[row + i:row + i + m, h * G:(h + 1) * G].reshape(m * G, -1) @ kh.T * case["d"] ** -0.5
                    x.masked_fill_(hidden, -math.inf)
                    l = torch.logsumexp(x, 1)
                    out["o"][row + i:row + i + m, h * G:(h + 1) * G] = (torch.exp(x - l[:, None]) @ vh).view(m, G, -1)
                    out["lse"][row + i:row + i + m, h * G:(h + 1) * G] = l.view(m, G)
            row += n
    if s["lse"] is None:
        out["lse"] = None
    return out
