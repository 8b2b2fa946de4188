"""The paged K/V cache in 16 and 8 bits at the limits of its arguments, without a GPU."""
import ctypes
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


FAKE = 0x7F0000001000      # never dereferenced: every call below ends in a check of its arguments


def _cache(**kw):
    c = dict(K_pool=FAKE, V_pool=FAKE, K_scale=FAKE, V_scale=FAKE, act_pool=None, block_table=FAKE, seq_len=FAKE, total_tokens=0,
             P_kv=10, P_act=0, n_act_used=0, block_tokens=16, max_blocks=1 << 12, n_kv_heads=8, format=hk.HK_KV_INT8)
    c.update(kw)
    return hk.hk_kv_cache(**c)


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,Hkv,T", [(4, 8, (1 << 22) - 15), (1, 1, (1 << 27) - 15), (64, 72, 29112), (1 << 16, 128, 1)])
def test_rows_that_one_store_holds(dh, B, Hkv, T):
    """B (T + 15) n_kv_heads <= 2^27: without k and v the call is refused for them up to there, for its size beyond."""
    assert B * (T + 15) * Hkv <= 1 << 27 < B * (T + 16) * Hkv
    shape, c = hk.make_shape(Hkv * dh, Hkv), _cache(n_kv_heads=Hkv)
    store = lambda T: hk.lib().hk_kv_store(ctypes.byref(shape), None, None, None, B, T, None, None, ctypes.byref(c), None)
    assert store(T) == hk.HK_ERR_NULL and store(T + 1) == hk.HK_ERR_SHAPE


@pytest.mark.parametrize("B,Hkv,L", [(4, 8, 1 << 23), (1, 1, 1 << 28), (128, 72, 29120)])
def test_rows_that_one_load_holds(B, Hkv, L):
    """B n_kv_heads ceil(L_cap / 32) <= 2^23, for both head dimensions."""
    for dh in (64, 128):
        shape, c = hk.make_shape(Hkv * dh, Hkv), _cache(n_kv_heads=Hkv)
        load = lambda L: hk.lib().hk_kv_load(ctypes.byref(shape), None, None, B, 0, L, ctypes.byref(c), None)
        assert load(L) == hk.HK_ERR_NULL and load(L + 1) == hk.HK_ERR_SHAPE


@pytest.mark.parametrize("T,H,splits,B", [(1, 8, 0, 1 << 20), (4, 64, 0, 1 << 17), (5, 64, 64, 1 << 12), (8, 64, 64, 1 << 12), (16, 64, 64, 1 << 11)])
def test_requests_that_one_attention_holds(T, H, splits, B):
    """8 K/V heads: all of 2^20 requests of one token; 32 rows: B T H = 2^25; 40 and 64 rows: 2^21 ranges, 128: 2^20
    (8192 tokens a request: a range has 4 tiles at least, which 64 pieces a request leave it)."""
    shape = hk.make_shape(H * 128, H, attn_splits=splits)
    size = lambda B: hk.lib().hk_kv_attn_workspace_bytes(ctypes.byref(shape), B, T, ctypes.byref(_cache(max_blocks=512 if splits else 8, total_tokens=B * 8192 if splits else 0)))
    assert size(B) > 0 and size(B + 1) == 0


def test_no_workgroup_walks_a_long_request_alone(tmp_path):
    exe = str(tmp_path / "kv_split_skew_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(ROOT, "tests", "host", "kv_split_skew_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
