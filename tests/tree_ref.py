"""Plain 64-bit forms of the tree and cache operators, on whatever device the
inputs are on, and their seeded inputs.  Imported by the tests of msa_tree.h and
msa_cache.h."""
from __future__ import annotations

import math
import random

import torch

BS = 16


def random_parents(r: random.Random, m: int, kind: str):
    if kind == "chain":
        return list(range(-1, m - 1))
    if kind == "star":
        return [-1] + [0] * (m - 1)
    if kind == "forest":  # several slots without a parent
        return [-1] + [r.choice((-1, r.randrange(i))) for i in range(1, m)]
    return [-1] + [r.randint(max(0, (i - 1) // 2 - 2), i - 1) for i in range(1, m)]


def ancestors(parents):
    """[m, m] truth: slot j is slot i or an ancestor of it."""
    m = len(parents)
    seen = torch.zeros(m, m, dtype=torch.bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            seen[i] = seen[p]
        seen[i, i] = True
    return seen


def mask_words(seen, words):
    """The int64 words of a truth matrix [m, m]."""
    m = seen.shape[0]
    out = torch.zeros(m, words, dtype=torch.int64)
    for i in range(m):
        for j in range(m):
            if seen[i, j]:
                v = 1 << (j % 64)
                out[i, j // 64] |= v - (1 << 64) if v >> 63 else v
    return out


def paged(lens, hkv, d, seed, device="cuda", extra_blocks=3):
    """Scattered caches of N(0, 1) values; the entries past a sequence's blocks are -1."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-L // BS) for L in lens]
    n = sum(counts) + extra_blocks
    table = torch.full((len(lens), max(1, max(counts, default=1))), -1, dtype=torch.int32)
    order = torch.randperm(n, generator=g).to(torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    k = torch.randn(n, hkv, BS, d, generator=g).to(torch.bfloat16)
    v = torch.randn(n, hkv, d, BS, generator=g).to(torch.bfloat16)
    return table.to(device), k.to(device), v.to(device)


def rows64(cache, table_row, n, head, is_v):
    blocks = cache[table_row[:-(-n // BS)].long(), head]
    blocks = blocks.transpose(1, 2) if is_v else blocks
    return blocks.reshape(-1, blocks.shape[-1])[:n].double()


def attention64(q, k, v, seen, scale):
    """o, lse and the bound's sum_j p_j |v_j| of rows q [n, d] over keys [L, d]; seen [n, L]."""
    hidden = ~seen.any(0)  # V that no row sees does not matter, whatever it holds
    v = torch.where(hidden[:, None], 0.0, v)
    x = (q.double() @ torch.where(hidden[:, None], 0.0, k).T) * scale
    x = torch.where(seen, x, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - torch.where(lse.isinf(), 0.0, lse)[:, None]), 0.0)
    return p @ v, lse, p @ v.abs()
