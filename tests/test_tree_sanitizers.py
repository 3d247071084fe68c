"""The planning of trees and of key weights under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only), with the instrumented build of
test_host_sanitizers.py: random plans of both kinds, and every refusal."""
import os
import subprocess
import sys

from test_host_sanitizers import ROOT, sanitized_builds  # noqa: F401

CODE = r"""
import random
import paper_2606_02964_amd as msa
r = random.Random(3)
for i in range(300):
    hq, hkv, d = r.choice(((8, 2, 128), (4, 4, 64), (64, 1, 64), (256, 1, 128), (32, 8, 128)))
    B = r.randint(0, 6)
    lens, indptr, start, length, tree = [], [0], [], [], []
    for b in range(B):
        at = r.choice((0, 0, 1, 17, 300, 9000))
        for _ in range(r.randint(0, 3)):
            n = r.choice((1, 2, 16, 63, 64, 65, 200, 1024))
            start.append(at); length.append(n); tree.append(r.randint(0, 1))
            at += n + r.choice((0, 1, 40))
        lens.append(at + r.randint(0, 5))
        indptr.append(len(start))
    blocks = max([1] + [-(-x // 16) for x in lens])
    shape = msa.make_shape(B, hq, hkv, d, blocks, max(1, blocks * B), 0.1)
    flags = msa.MSA_PLAN_HOST_ONLY
    p = msa.msa_plan_tree(shape, lens, indptr, start, length, r.choice((tree, None)), flags=flags)
    msa.msa_plan_tree_info(p); p.info(); msa.msa_plan_export(p)
    q = msa.msa_plan(shape, lens, indptr, start, length, flags=flags)
    q.info()
    if start:
        bad = list(tree); bad[r.randrange(len(bad))] = 7
        try:
            msa.msa_plan_tree(shape, lens, indptr, start, length, bad, flags=flags)
            raise SystemExit("accepted")
        except msa.MsaError:
            pass
shape = msa.make_shape(1, 64, 8, 128, 5000, 5000, 0.1)
msa.msa_plan(shape, [80000], [0, 1], [0], [70000], flags=msa.MSA_PLAN_HOST_ONLY)
print("planned")
"""


def test_tree_and_weight_plans_are_clean(sanitized_builds):  # noqa: F811
    lib, _, asan = sanitized_builds
    env = dict(os.environ, MSA_LIBRARY=lib, LD_PRELOAD=asan, PYTHONDONTWRITEBYTECODE="1",
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    text = res.stdout + res.stderr
    assert "AddressSanitizer" not in text and "runtime error:" not in text, text[-4000:]
    assert res.returncode == 0 and "planned" in res.stdout, text[-4000:]
