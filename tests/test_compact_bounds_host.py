"""msa_kv_compact where there is nothing that could move (no GPU).  The addresses given are never read."""
import ctypes

import pytest

import paper_2606_02964_amd as msa

P = 4096  # an address


@pytest.mark.parametrize("max_count", [1, 64, 65, 5000])
@pytest.mark.parametrize("shape", [dict(max_blocks_per_seq=0), dict(num_blocks=0), dict(num_seqs=0)])
def test_a_table_without_entries_is_not_read(shape, max_count):
    """No sequence has a position, so no list can hold a move: the call returns without a launch, whatever counts and
    lists there are."""
    a = dict(num_seqs=2, num_q_heads=8, num_kv_heads=2, head_dim=128, max_blocks_per_seq=200, num_blocks=400, scale=0.1)
    a.update(shape)
    sh = msa.make_shape(**a)
    for base in (P, None):
        assert msa._lib.msa_kv_compact(ctypes.byref(sh), base, P, 50, 0, max_count, P, P, P, P, None) == msa.MSA_OK
