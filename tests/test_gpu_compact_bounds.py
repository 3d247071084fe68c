"""Compaction at the ends of the block table, lists of either kernel: up to 64 entries, and more (GPU only).  Against
the element by element form of test_gpu_cache.py."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

from test_gpu_cache import check_compact, pick  # noqa: E402


@pytest.mark.parametrize("n", [64, 65, 415, 700])
@pytest.mark.parametrize("back", [1, 15, 16, 20, 33])
def test_a_base_before_the_first_position(n, back):
    """Every entry i whose destination base + i is in the table moves, those of i >= the table's positions too."""
    idx = list(range(n // 2)) + list(range(n // 2 + 5, n + 5))
    for cap in (n + 5 - back, n - back, n // 2 + 9):  # the last move's source is the last position, or behind it
        check_compact([cap], [-back], [len(idx)], [[idx, idx]])


@pytest.mark.parametrize("n", [60, 300])
def test_a_base_near_and_past_the_last_position(n):
    idx = list(range(3)) + list(range(5, n + 2))
    for base in (1, 16, 100, n - 1, n, n + 40, 2 ** 31 - 1):
        check_compact([n + 20], [base], [len(idx)], [[idx, idx]])


def test_long_lists_skip_what_lies_outside():
    """Blocks outside the cache as sources and as destinations, counts past the list, positions past the table."""
    r = random.Random(1)
    lens = [700, 700, 700, 700]
    idx = pick(r, 700, 333)
    check_compact(lens, [0, 3, 16, -18], [len(idx), 1 << 30, -4, len(idx)], [[idx, idx]] * 4,
                  spoil=[(0, 1, -1), (0, 20, 1 << 30), (1, 0, -5), (1, 43, -1), (3, 7, -2 ** 31), (3, 30, 2 ** 31 - 1)])
    far = pick(r, 700, 200) + list(range(5000, 5200))
    check_compact([700], [0], [len(far)], [[far, far]])


@pytest.mark.parametrize("entries", [40, 200])
def test_lists_of_two_parts_of_one_sequence(entries):
    """Lists whose places lie side by side in a block, each of a row of the table that names the same blocks."""
    from tree_ref import paged
    from test_gpu_cache import compact_ref
    import paper_2606_02964_amd as msa
    r = random.Random(2)
    table, k, v = paged([1000], 2, 128, 3)
    base = [5, 5 + 333, 5 + 333 + 300]
    lists = [pick(r, m, min(entries, m)) for m in (333, 300, 61)]
    rows = table.repeat(3, 1).contiguous()
    shape = msa.make_shape(3, 2, 2, 128, rows.shape[1], k.shape[0], 1.0)
    index = torch.full((3, entries), 1 << 30, dtype=torch.int32)
    for b, x in enumerate(lists):
        index[b, :len(x)] = torch.tensor(x, dtype=torch.int32)
    count = [len(x) for x in lists]
    want_k, want_v = compact_ref(k.cpu(), v.cpu(), rows.cpu(), base, [[x, x] for x in lists], count, rows.shape[1] * 16)
    msa.msa_kv_compact(shape, torch.tensor(base, dtype=torch.int32).cuda(), index.cuda(),
                       torch.tensor(count, dtype=torch.int32).cuda(), rows, k, v)
    torch.cuda.synchronize()
    assert torch.equal(k.cpu().view(torch.int16), want_k.view(torch.int16))
    assert torch.equal(v.cpu().view(torch.int16), want_v.view(torch.int16))
