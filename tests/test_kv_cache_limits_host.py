"""The paged K/V cache in 16 and 8 bits at the limits of its arguments, without a GPU."""
import os
import subprocess

import pytest
import torch

from paper_2501_01792_amd import binding as hk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("Hkv,dh,width", [(2, 64, 64), (2, 64, 127), (2, 64, 256), (8, 128, 4096), (1, 128, 64)])
def test_checkpoint_rows_are_as_wide_as_the_layer(Hkv, dh, width):
    """kv_store writes rows of n_kv_heads * dh into act_pool: a narrower pool would be left behind its end, and a wider one (a layer
    whose query heads share K/V heads) has no ACT blocks."""
    pool, table, lens = torch.zeros(3, Hkv, 16, dh).half(), torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="act_pool"):
        hk.make_kv_cache(pool, pool, table, lens, 16, act_pool=torch.zeros(2, 16, width).half())
    with pytest.raises(TypeError):                         # the right width comes as far as the check for a GPU
        hk.make_kv_cache(pool, pool, table, lens, 16, act_pool=torch.zeros(2, 16, Hkv * dh).half())

    with pytest.raises(TypeError):                         # no blocks: nothing that could be too narrow
        hk.make_kv_cache(pool, pool, table, lens, 16, act_pool=torch.zeros(0, 16, width).half())


def test_pieces_of_sums_beyond_32_bits(tmp_path):
    exe = str(tmp_path / "kv_split_far_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(ROOT, "tests", "host", "kv_split_far_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
