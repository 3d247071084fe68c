"""Code-generation checks of the tree and cache kernels (CPU only: hipcc
cross-compiles), as test_kernel_isa.py makes them of the others:

* no kernel spills registers or uses scratch memory (the attention kernels may
  push two scalar registers into lanes of a vector register, once per workgroup);
* the tree kernels keep two waves per SIMD and read MFMA operands ahead, the key
  weights' kernels two and three waves;
* the key weights' exponentials stand beside the MFMAs of the next tile: left to
  itself the compiler moves them all behind the MFMAs.
"""
import os
import re
import subprocess

import pytest

from paper_2606_02964_amd import build as B
from test_kernel_isa import _body, _hipcc, _resources

SOURCES = ("tree.hip", "verify.hip", "weights.hip", "select.hip", "compact.hip")


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    cc, out, tmp, running = _hipcc(), {}, tmp_path_factory.mktemp("isa"), {}
    for src in SOURCES:
        asm = tmp / (src + ".s")
        cmd = [cc, *B.common_flags(), "--cuda-device-only", "-S", "-Rpass-analysis=kernel-resource-usage",
               os.path.join(B.CSRC, src), "-o", str(asm)]
        running[src] = (asm, subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE, text=True))
    for src, (asm, p) in running.items():
        err = p.communicate()[1]
        assert p.returncode == 0, err[-2000:]
        out[src] = (asm.read_text(), err)
    return out


@pytest.mark.parametrize("src", SOURCES)
def test_no_spills_or_scratch(compiled, src):
    kernels = _resources(compiled[src][1])
    assert kernels, "no resource remarks parsed"
    for name, r in kernels.items():
        assert r.get("VGPRs Spill", 0) == 0 and r.get("SGPRs Spill", 0) <= 2, (name, r)
        assert r.get("ScratchSize", 0) == 0, (name, r)


def test_occupancy(compiled):
    tree = {k: v for k, v in _resources(compiled["tree.hip"][1]).items() if "mask" not in k}
    assert len(tree) == 16  # d in {64, 128} x four kernels x {bf16 weights, precise weights}
    assert all(r["Occupancy"] >= 2 for r in tree.values())
    weights = _resources(compiled["weights.hip"][1])
    assert all(r["Occupancy"] >= 3 for k, r in weights.items() if "stream" in k)
    assert all(r["Occupancy"] >= 2 for k, r in weights.items() if "tiles" in k)
    assert all(r["Occupancy"] >= 4 for r in _resources(compiled["select.hip"][1]).values())
    assert all(r["Occupancy"] >= 4 for r in _resources(compiled["compact.hip"][1]).values())


def test_operand_reads_run_ahead(compiled):
    asm, remarks = compiled["tree.hip"]
    names = [k for k in _resources(remarks) if re.search(r"msa_tree_kernel|msa_tree_helped_kernel", k)]
    assert len(names) == 12
    for name in names:
        waits = re.findall(r"s_waitcnt lgkmcnt\((\d+)\)", _body(asm, name))
        assert sum(1 for n in waits if int(n) >= 1) >= 0.5 * len(waits), name


def test_weights_beside_mfmas(compiled):
    asm, remarks = compiled["weights.hip"]
    for name in (k for k in _resources(remarks) if "tiles" in k):
        per_tile = 17 if "ILi128E" in name else 9
        body = _body(asm, name).split("s_barrier")[1:]
        pipelined = [b for b in body if len(re.findall(r"v_mfma_f32_32x32x16_bf16", b)) == per_tile
                     and len(re.findall(r"v_exp_f32", b)) == 32]
        assert len(pipelined) >= 2, name
        for b in pipelined:  # no run of exponentials as long as a tile's without an MFMA between them
            ops = re.findall(r"v_mfma_f32_32x32x16_bf16|v_exp_f32", b)
            longest = run = 0
            for op in ops:
                run = run + 1 if op == "v_exp_f32" else 0
                longest = max(longest, run)
            assert longest <= 8, (name, longest)
