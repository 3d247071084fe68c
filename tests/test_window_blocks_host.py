"""Blocks that a plan of msa_plan_window reads, as the read-me's function gives them: the block-table check asks
for these and no others, and every block that a work item loads is one of them."""
import os
import random
import re

import numpy as np
import pytest

import paper_2606_02964_amd as msa

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BS, STEP = 16, 64


def readme_function():
    text = open(os.path.join(ROOT, "README.md"), encoding="utf-8").read()
    (block,) = [b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "def blocks_read" in b]
    names = {}
    exec(block, names)
    return names["blocks_read"]


def layout(r):
    """(lengths, indptr, starts, lengths of segments, first and last row of each sequence)."""
    lens, indptr, start, length, ends = [], [0], [], [], []
    for _ in range(r.randint(1, 3)):
        at, first = r.choice((0, 3, 100, 800, 2000)), len(start)
        for _ in range(r.randint(0, 4)):
            n = r.choice((1, 1, 4, 16, 30, 64, 150))
            start.append(at)
            length.append(n)
            at += n + r.choice((0, 1, 15, 96, 500, 1500))
        ends.append((start[first], start[-1] + length[-1] - 1) if len(start) > first else None)
        lens.append(at + r.randint(1, 40))
        indptr.append(len(start))
    return lens, indptr, start, length, ends


def loaded(pos, item, window, sinks):
    """The blocks that a work item's steps load, and those that stand in for ones without a visible key."""
    _, _, row0, _, lo, hi, _, _ = item
    first = max(0, int(pos[row0]) - window + 1)
    head = -(-sinks // STEP) * STEP
    skip = max(0, first // STEP * STEP - head)
    blocks = set()
    for v in range(lo, hi, BS):
        b = (v if v < head else v + skip) // BS
        blocks.add(first // BS if -(-sinks // BS) <= b < first // BS else b)
    return blocks


@pytest.mark.parametrize("seed", range(8))
def test_blocks_of_the_read_me(seed):
    blocks_read, r = readme_function(), random.Random(seed)
    gaps = 0
    for _ in range(10):
        lens, indptr, start, length, ends = layout(r)
        window, sinks = r.choice((1, 8, 40, 64, 100, 700)), r.choice((0, 1, 4, 20, 64, 200))
        if window > max([b for e in ends if e for b in e] + [0]):
            continue  # (a causal plan)
        MB = max(-(-x // BS) for x in lens)
        shape = msa.make_shape(len(lens), *r.choice(((8, 2, 128), (4, 4, 64), (32, 8, 128))), MB, MB * len(lens), 0.1)
        flags = r.choice((0, msa.MSA_PLAN_TILE_ROWS_32, msa.MSA_PLAN_TILE_ROWS_128, msa.MSA_PLAN_TILE_ROWS_256))
        plan = msa.msa_plan_window(shape, lens, indptr, start, length, window, sinks,
                                   kv_split_tokens=r.choice((0, 0, 64)), flags=flags | msa.MSA_PLAN_HOST_ONLY)
        promised = [blocks_read(*e, window, sinks) if e else set() for e in ends]
        pos, work, _ = msa.msa_plan_export(plan)
        for item in work.tolist():
            assert loaded(pos, item, window, sinks) <= promised[item[0]]
        table = np.full((len(lens), MB), -1, dtype=np.int32)
        for b, blocks in enumerate(promised):
            table[b, sorted(blocks)] = 0
        msa.msa_check_block_table(plan, table)
        for b, blocks in enumerate(promised):
            for i in sorted(blocks)[::max(1, len(blocks) // 9)]:
                table[b, i] = -1
                with pytest.raises(msa.MsaError, match=f"sequence {b}, logical block {i} "):
                    msa.msa_check_block_table(plan, table)
                table[b, i] = 0
            # blocks between segments that no row sees are of the promised ones too
            seen = {j // BS for k in range(indptr[b], indptr[b + 1]) for p in range(start[k], start[k] + length[k])
                    for j in (max(0, p - window + 1), p)} if ends[b] else set()
            gaps += len({i for i in blocks if i * BS >= sinks} - seen) > 0
    assert gaps > 0


def test_rows_behind_a_gap():
    """Rows 800 .. 803 and 900 .. 903 with 8 keys each: one tile over both, whose items load the blocks between."""
    shape = msa.make_shape(1, 8, 2, 128, 60, 60, 0.1)
    plan = msa.msa_plan_window(shape, [960], [0, 2], [800, 900], [4, 4], 8, 0, flags=msa.MSA_PLAN_HOST_ONLY)
    table = np.full((1, 60), -1, dtype=np.int32)
    table[0, sorted(readme_function()(800, 903, 8, 0))] = 0
    msa.msa_check_block_table(plan, table)
    assert (table[0] == 0).nonzero()[0].tolist() == list(range(49, 57))
    pos, work, _ = msa.msa_plan_export(plan)
    assert set().union(*(loaded(pos, item, 8, 0) for item in work.tolist())) == set(range(49, 57))
