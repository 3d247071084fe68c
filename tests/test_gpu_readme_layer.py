"""The read-me's blocks of rotary positions, the 8-bit cache and windows, run as they stand."""
import os
import re

import pytest
import torch

import paper_2606_02964_amd as msa
from serve_ref import BS, Layout, normal, o_bound, rotate

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def block(holds):
    blocks = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md"), encoding="utf-8").read(), re.S)
    (found,) = [b for b in blocks if holds in b]
    return found


def test_blocks():
    lay = Layout([(6000, [(4990, 20), (5990, 10)]), (700, [(100, 300)])], 32, 8, 128, seed=1)
    names = dict(msa=msa, torch=torch, layers=range(2), shape=lay.shape(msa), seq_kv_len=lay.lens, seg_indptr=lay.indptr,
                 seg_start=lay.start, seg_len=lay.length, block_table=lay.table, NB=lay.num_blocks, max_len=6000,
                 end=torch.tensor(lay.lens, dtype=torch.int32, device="cuda"))
    names.update(q=normal(1, lay.rows, 32, 128), q_rotated=torch.empty(lay.rows, 32, 128, dtype=torch.bfloat16, device="cuda"),
                 k_new=normal(2, lay.rows, 8, 128), v_new=normal(3, lay.rows, 8, 128),
                 k_cache=normal(4, lay.num_blocks, 8, BS, 128), v_cache=normal(5, lay.num_blocks, 8, 128, BS),
                 o=torch.empty(lay.rows, 32, 128, dtype=torch.bfloat16, device="cuda"), lse=torch.empty(lay.rows, 32, device="cuda"))
    exec(block("msa_plan_window"), names)
    plan = names["plan"]
    names["ws"] = torch.empty(max(1, plan.info()["workspace_bytes"]), dtype=torch.uint8, device="cuda")
    exec(block("msa_rope_freqs"), names)
    torch.cuda.synchronize()

    def check():
        ref = lay.attend(names["q_rotated"], names["k_cache"], names["v_cache"], 4096, 4)
        assert ((names["o"].double() - ref[0]).abs() <= o_bound(ref[0], ref[2])).all()
        assert (names["lse"].double() - ref[1]).abs().max() <= 2.5e-4
    check()
    want = rotate(names["q"], lay.pos, torch.from_numpy(names["freq"]).cuda(), 0, names["amplitude"])
    assert ((names["q_rotated"].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * 16).all()
    kb = names["k_cache"].clone()
    exec(block("msa_fp8_read"), names)  # a fresh cache: zeros but for the rows
    torch.cuda.synchronize()
    check()  # over the cache as it was read back
    blk, at = lay.places()
    far = (names["k_cache"][blk, :, at].double() - kb[blk, :, at].double()).abs()
    top = kb[blk, :, at].double().abs()
    # e4m3 and the bf16 cache's own rounding: 2^-4 and 2^-8 of a number, and half the smallest step below
    assert (far <= top * (2.0 ** -4 + 2.0 ** -7) + top.amax(-1, keepdim=True) * 2.0 ** -17).all()
    assert int((names["v_cache"] != 0).sum()) > 0
