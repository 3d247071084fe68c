"""The planning of windows under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only), with the
instrumented build of test_host_sanitizers.py: random plans, block tables, and the largest arguments."""
import os
import subprocess
import sys

from test_host_sanitizers import ROOT, sanitized_builds  # noqa: F401

CODE = r"""
import random
import numpy as np
import paper_2606_02964_amd as msa
r = random.Random(7)
BIG = (1 << 31) - 1
for i in range(250):
    hq, hkv, d = r.choice(((8, 2, 128), (4, 4, 64), (64, 1, 64), (256, 1, 128), (32, 8, 128)))
    B = r.randint(0, 5)
    lens, indptr, start, length = [], [0], [], []
    for b in range(B):
        at = r.choice((0, 0, 1, 17, 300, 9000))
        for _ in range(r.randint(0, 3)):
            n = r.choice((1, 2, 16, 63, 64, 65, 200, 3000))
            start.append(at); length.append(n)
            at += n + r.choice((0, 1, 40, 5000))
        lens.append(at + r.randint(0, 5))
        indptr.append(len(start))
    blocks = max([1] + [-(-x // 16) for x in lens])
    shape = msa.make_shape(B, hq, hkv, d, blocks, max(1, blocks * B), 0.1)
    window = r.choice((1, 2, 63, 64, 65, 1000, 8000, BIG - 1, BIG))
    sinks = r.choice((0, 1, 4, 64, 65, 5000, BIG - 63, BIG))
    p = msa.msa_plan_window(shape, lens, indptr, start, length, window, sinks, kv_split_tokens=r.choice((0, 0, 64, 1024)),
                            flags=msa.MSA_PLAN_HOST_ONLY)
    p.info(); msa.msa_plan_export(p)
    msa.msa_check_block_table(p, np.zeros((max(1, B), blocks), np.int32))
shape = msa.make_shape(1, 64, 8, 128, BIG // 16, 5000, 0.1)  # positions next to the last one of 32 bits
L = BIG // 16 * 16
for window, sinks in ((100, BIG), (BIG, 3), (1, 0), (70, L), (L - 70, 65)):
    p = msa.msa_plan_window(shape, [L], [0, 2], [L - 9000, L - 65], [20, 65], window, sinks, flags=msa.MSA_PLAN_HOST_ONLY)
    assert p.info()["total_q"] == 85
print("planned")
"""


def test_window_plans_are_clean(sanitized_builds):  # noqa: F811
    lib, _, asan = sanitized_builds
    env = dict(os.environ, MSA_LIBRARY=lib, LD_PRELOAD=asan, PYTHONDONTWRITEBYTECODE="1",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    text = res.stdout + res.stderr
    assert "AddressSanitizer" not in text and "runtime error:" not in text, text[-4000:]
    assert res.returncode == 0 and "planned" in res.stdout, text[-4000:]
