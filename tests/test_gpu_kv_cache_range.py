"""Attention over 8-bit caches whose rows of V lie as far apart as their types allow: every token counts in the denominator,
whatever its V is.  kv_store gives a row of zeros the scale 2^-100; bf16 rows reach 2^127.  Against the oracle in 64 bits, held
to the bound of the ordinary cases (which is relative to the sum of p |v|)."""
import numpy as np
import pytest
import torch

from paper_2501_01792_amd import binding as hk
from test_gpu_kv_cache import Cache, check_attention, normal

pytestmark = pytest.mark.gpu


def spread(c, r, tokens, power):
    """Rows of V of those tokens times 2^power (None: rows of zeros, as kv_store writes them)."""
    for t in tokens:
        e = int(c.table[r, t // c.bt])
        if power is None:
            c.pools[1].view(torch.int8)[e, :, t % c.bt] = 0
            c.scales[1][e, :, t % c.bt] = 2.0 ** -100
        else:
            c.scales[1][e, :, t % c.bt] *= 2.0 ** power


PLACES = {
    "by turns": lambda n: range(0, n, 2),
    "first": lambda n: range(n // 2),                      # whole tiles, pieces and wavefronts' shares of them
    "last": lambda n: range(n // 2, n),
    "all but one": lambda n: [t for t in range(n) if t != n // 3],
}


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("place", list(PLACES))
@pytest.mark.parametrize("small,large", [(None, 0), (None, 34), (None, 60), (None, 110), (-60, 62), (-30, 40)])
@pytest.mark.parametrize("T,dh", [(0, 64), (0, 128), (5, 64), (20, 64), (20, 128), (36, 64)])
def test_every_token_counts(form, place, small, large, T, dh):
    """T = 0: one token; 5 nodes: the form of up to 32 rows, 20 and 36 nodes of 2 query heads a K/V head: of more."""
    lens, H, Hkv, bt = [900, 70], 4, 2, 16
    c = Cache(200 + dh, form, "bf16", lens, Hkv, dh, bt)
    for r, n in enumerate(lens):
        few = set(PLACES[place](n))
        spread(c, r, few, small)
        spread(c, r, [t for t in range(n) if t not in few], large)
    q = normal(201, 2, max(T, 1), H, dh, dtype="bf16")
    k, v = (normal(202 + i, 2, T, Hkv, dh, dtype="bf16") for i in range(2))
    for splits in (0, 1, 3):
        if T:
            check_attention("spread", c, q, k, v, None, None, hk.kv_tree_attn(q, k, v, c.handle, attn_splits=splits))
        else:
            check_attention("spread", c, q, None, None, None, None, hk.kv_decode_attn(q[:, 0].contiguous(), c.handle, attn_splits=splits)[:, None])


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("T", [5, 20])
@pytest.mark.parametrize("cache,nodes", [(110, 0), (118, 0), (60, -60), (-60, 60), (None, 60), (None, 100), (None, -60), (-90, 30)])
def test_nodes_and_tokens_far_apart(form, T, cache, nodes):
    """V of the nodes and V of the cache at opposite ends of bf16."""
    lens, H, Hkv, dh, bt = [300, 70, 0, 1], 4, 2, 64, 16
    c = Cache(210, form, "bf16", lens, Hkv, dh, bt)
    for r, n in enumerate(lens):
        spread(c, r, range(n), cache)
    q, k, v = normal(211, 4, T, H, dh, dtype="bf16"), normal(212, 4, T, Hkv, dh, dtype="bf16"), normal(213, 4, T, Hkv, dh, dtype="bf16") * 2.0 ** nodes
    v[:, 1] = 0
    for splits in (0, 1, 3):
        check_attention("nodes", c, q, k, v, None, None, hk.kv_tree_attn(q, k, v, c.handle, attn_splits=splits))


@pytest.mark.parametrize("T", [1, 20])
@pytest.mark.parametrize("dtype,power", [("f16", 12), ("bf16", 12), ("bf16", 100)])
@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_many_tokens_of_small_weight(form, dtype, power, T):
    """60000 rows of zeros of weight 2^-18 each beside one row of large V: together a fifth of the denominator."""
    n, H, Hkv, dh, bt = 60001, 2, 1, 64, 1024
    c = Cache(220, form, dtype, [n], Hkv, dh, bt)
    one = 64 if form == "int8" else 0x38                   # the code of 64, of 1
    c.pools[0].view(torch.int8)[:] = one
    c.scales[0][:] = 2.0 ** -6 if form == "int8" else 1.0  # K of ones
    spread(c, 0, range(n), None)
    e, at = int(c.table[0, 40000 // bt]), 40000 % bt
    c.pools[0].view(torch.int8)[e, :, at] = 0              # a score of 0, the others' -18 log 2
    c.pools[1].view(torch.int8)[e, :, at] = one
    c.scales[1][e, :, at] = 2.0 ** (power - 6 if form == "int8" else power)
    q = torch.full((1, T, H, dh), -18 * np.log(2) / 8, dtype=torch.float64).to(torch.float16 if dtype == "f16" else torch.bfloat16).cuda()
    for splits in (0, 1, 3):
        if T == 1:
            got = hk.kv_decode_attn(q[:, 0].contiguous(), c.handle, attn_splits=splits)[:, None]
            check_attention("many", c, q, None, None, None, None, got)
        else:
            k = torch.zeros(1, T, Hkv, dh, dtype=q.dtype, device="cuda")
            none = torch.zeros(T, dtype=torch.int64, device="cuda")      # the nodes are seen by nobody
            got = hk.kv_tree_attn(q, k, k, c.handle, mask=none, attn_splits=splits)
            check_attention("many", c, q, k, k, none.cpu(), None, got)
