"""Key weights where 32 is no multiple of the query heads of a KV head, so that tiles of 32 (row, head) pairs begin and
end within a row, and of plans with many items (GPU only).  Bar and reference are those of test_gpu_cache.py."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # collected on a CPU-only host with -m gpu
    pytest.skip("no GPU visible", allow_module_level=True)

from test_gpu_cache import Weights  # noqa: E402
from tree_ref import rows64  # noqa: E402

GROUPS = [(28, 4, 128), (12, 4, 64), (6, 1, 128), (10, 2, 64), (24, 2, 128), (24, 1, 64), (33, 1, 128), (100, 1, 64),
          (255, 1, 64)]


@pytest.mark.parametrize("heads", GROUPS)
def test_lengths(heads):
    ends = [1, 2, 3, 5, 11, 16, 17, 31, 33, 64, 65, 100, 255, 256, 257, 300]
    w = Weights([[(0, n)] for n in ends] + [[]] + [[(n - 1, 1)] for n in ends], heads, more=3, q_pad=8)
    w.check(w.run())


@pytest.mark.parametrize("heads", GROUPS)
def test_segments(heads):
    r = random.Random(3)
    segs = []
    for L in (900, 513, 64, 2000, 1300):
        a = sorted(r.sample(range(0, L, 7), 6))
        segs.append([(a[0], a[1] - a[0]), (a[2], 1), (a[3], a[4] - a[3]), (L - 2, 2)] if L > 100 else [(L - 1, 1)])
    w = Weights(segs, heads)
    w.check(w.run())
    assert torch.equal(w.run(), w.run())


@pytest.mark.parametrize("heads", [(28, 4, 128), (12, 4, 64), (10, 2, 64)])
def test_many_tiles_in_parts(heads):
    w = Weights([[(20000, 1)], [(0, 2500)], [(7, 1)], [(5000, 701)], [(1000, 3), (1100, 90), (1500, 400)]], heads)
    w.check(w.run())


@pytest.mark.parametrize("heads", [(32, 8, 128), (7, 1, 64)])
def test_a_long_prompt(heads):
    """Items by the hundred, sorted by counting; sums of some keys, every row."""
    n = 17000
    w = Weights([[(5, 40)], [(0, n)], [(0, 2000), (9000, 100), (30000, 3)]], heads)
    got = w.run(accumulate=False)
    torch.cuda.synchronize()
    r, G = random.Random(4), w.hq // w.hkv
    keys = sorted({0, 1, 255, 256, 257, n - 258, n - 257, n - 256, n - 2, n - 1} | set(r.sample(range(n), 40)))
    at = torch.tensor(keys, device="cuda")
    q = w.q[40:40 + n, :w.hq * w.d].reshape(n, w.hq, w.d)
    seen = torch.arange(n, device="cuda")[:, None] >= at[None, :]
    for h in range(w.hkv):
        k = rows64(w.k, w.table[1], n, h, False)[at]
        want = torch.zeros(len(keys), dtype=torch.float64, device="cuda")
        for i in range(h * G, h * G + G):
            x = (q[:, i].double() @ k.T) * w.scale - w.lse[40:40 + n, i, None].double()
            want += torch.where(seen, torch.exp(x), 0.0).sum(0)
        assert ((got[1, h, at].double() - want).abs() <= 2.0 ** -17 * want).all(), h
    total = got[1, :, :n].double().sum(1)
    assert ((total / (n * G) - 1).abs() <= 2.0 ** -16).all()
    assert torch.equal(got[1, :, n:], w.before[1, :, n:])
