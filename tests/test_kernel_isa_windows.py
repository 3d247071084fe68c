"""Code-generation checks of the window, 8-bit cache and rotary kernels (CPU only: hipcc
cross-compiles), as test_kernel_isa.py makes them of the others:

* no vector register goes to scratch memory; scalar registers go to lanes of vector ones only in
  the kernels that have both a window and an 8-bit cache, in the write kernel's 8-bit forms, which
  hold most arguments (there once a workgroup), and one of an item's end in the 8-bit rows kernel;
* tiles and rows keep two waves per SIMD, and their LDS lets two workgroups of 128-row tiles stay on a CU;
* MFMA operand reads run ahead, and the pipelined step of an 8-bit tile has its conversions among its MFMAs;
* numbers go to and from 8 bits by the conversion instructions.
"""
import os
import re
import subprocess

import pytest

from paper_2606_02964_amd import build as B
from test_kernel_isa import _body, _hipcc, _resources

SOURCES = ("window.hip", "fp8.hip", "rope.hip")


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


@pytest.mark.parametrize("src,kernels", [("window.hip", 16), ("fp8.hip", 34), ("rope.hip", 10)])
def test_registers(compiled, src, kernels):
    found = _resources(compiled[src][1])
    assert len(found) == kernels
    for name, r in found.items():
        assert r.get("VGPRs Spill", 0) == 0 and r.get("ScratchSize", 0) == 0, (name, r)
        most = 24 if "Fp8" in name and "Window" in name else 20 if "rope" in name else 1 if "Fp8" in name and "rows" in name else 0
        assert r.get("SGPRs Spill", 0) <= most, (name, r)


@pytest.mark.parametrize("src", SOURCES[:2])
def test_occupancy(compiled, src):
    for name, r in _resources(compiled[src][1]).items():
        assert r["Occupancy"] >= (4 if "read" in name else 2), (name, r)
        lds = r.get("LDS Size", 0)
        assert lds <= (160 << 10) // 2, (name, r)


@pytest.mark.parametrize("src", SOURCES[:2])
def test_operand_reads_run_ahead(compiled, src):
    asm, remarks = compiled[src]
    names = [k for k in _resources(remarks) if "tiles" in k]
    assert len(names) == (12 if src == "window.hip" else 24)
    for name in names:
        waits = re.findall(r"s_waitcnt lgkmcnt\((\d+)\)", _body(asm, name))
        assert sum(1 for n in waits if int(n) >= 1) >= 0.4 * len(waits), name


def test_conversions(compiled):
    asm, remarks = compiled["fp8.hip"]
    for name in _resources(remarks):
        body = _body(asm, name)
        assert "v_cvt_scalef32_pk_bf16_fp8" in body, name
        if "tiles" in name:  # (the write to the rings in a step with MFMAs)
            assert "v_cvt_scalef32_f32_fp8" in body, name
            if "ELb1ELb1EEE" in name or "ELb0ELb1EEE" in name:
                continue  # helpers convert: no MFMA is beside them
            between = [b for b in re.split(r"v_mfma_f32_32x32x16_bf16", body) if "v_cvt_scalef32_f32_fp8" in b and b.count("\n") < 200]
            assert len(between) >= 2, name  # the two steps of the paired loop
    asm, remarks = compiled["rope.hip"]
    for name in _resources(remarks):
        assert ("v_cvt_pk_fp8_f32" in _body(asm, name)) == ("Lb1E" in name), name
