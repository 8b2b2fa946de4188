"""The paged K/V cache in 16 and 8 bits without a GPU: pins of its oracle, the cut of the tokens, the argument checks of the
calls and of the binding."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from oracle import kv_oracle as ko
from paper_2501_01792_amd import binding as hk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000001000      # never dereferenced: every call below must fail validation first


# ------------------------------------------------------------------ oracle pins
def test_e4m3_codes_by_hand():
    v = ko.e4m3_values()
    assert v[0x38] == 1.0 and v[0x7E] == 448.0 and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6 and np.isnan(v[0x7F]) and v[0xB8] == -1.0
    y = np.array([0.0, 1.0, 1.0625, 1.1875, 448.0, 463.9, 2.0 ** -10, 3 * 2.0 ** -10, -300.0])
    # ties go to the even mantissa: 1.0625 lies between 1 and 1.125, 1.1875 between 1.125 and 1.25
    assert [ko._E4M3[c] for c in ko.e4m3_code(y)] == [0.0, 1.0, 1.0, 1.25, 448.0, 448.0, 0.0, 2.0 ** -8, -288.0]
    codes = np.delete(np.arange(256), [127, 255])
    assert (ko.e4m3_code(v[codes]) == codes).all()
    torch_v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert (np.isnan(v) == np.isnan(torch_v)).all() and (v[codes] == torch_v[codes]).all()


@pytest.mark.parametrize("form", ["int8", "e4m3"])
def test_quantised_rows_are_half_a_step_off_at_most(form):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((200, 64)) * 10.0 ** rng.uniform(-5, 3, (200, 1))).astype(np.float16).astype(np.float32)
    code, scale = ko.quantise(x, form)
    err = np.abs(ko.dequantise(code, scale, form) - x)
    step = np.full_like(x, 1.0) if form == "int8" else np.maximum(2.0 ** (np.floor(np.log2(np.maximum(np.abs(x / scale[:, None]), 2.0 ** -6))) - 3), 2.0 ** -9)
    assert (err <= (0.5 * step + 2.0 ** -20 * 448) * scale[:, None]).all()
    assert (np.abs(ko.dequantise(code, scale, form)).max(1) >= np.abs(x).max(1) * (1 - 2.0 ** -20)).all()    # the largest is exact
    code, scale = ko.quantise(np.zeros((1, 64)), form)
    assert scale[0] == ko.LEAST_SCALE and (ko.dequantise(code, scale, form) == 0).all()
    bad = np.ones((2, 64), np.float32)
    bad[0, 5], bad[1, 7] = np.inf, np.nan
    code, scale = ko.quantise(bad, form)
    assert np.isnan(scale).all() and (code == 0).all()


def test_attention_oracle_by_hand():
    K, V = np.array([[1.0, 0.0], [1.0, 0.0]]), np.array([[2.0, 4.0], [4.0, -4.0]])
    out, size, most, peak = ko.attend(np.array([3.0, 1.0]), K, V, np.array([True, True]), 0.5)
    assert np.allclose(out, [3.0, 0.0]) and np.allclose(size, [3.0, 4.0]) and most == 1.5 and peak == 2.0
    assert (ko.attend(np.ones(2), K, V, np.array([False, True]), 1.0)[0] == [4.0, -4.0]).all()
    assert (ko.attend(np.ones(2), K, V, np.array([False, False]), 1.0)[0] == 0).all()


# ------------------------------------------------------------------ masks
def test_tree_mask():
    m = hk.tree_mask([-1, 0, 0, 2, -1]).tolist()
    assert m == [0b1, 0b11, 0b101, 0b1101, 0b10000]
    chain = hk.tree_mask(list(range(-1, 63)))
    assert chain[62].item() == (1 << 63) - 1 and chain[63].item() == -1 and chain.dtype == torch.int64
    assert hk.tree_mask([]).numel() == 0
    for bad in ([0], [-1, 1], [-2], [-1, 5]):
        with pytest.raises(ValueError):
            hk.tree_mask(bad)
    with pytest.raises(ValueError):
        hk.tree_mask([-1] * 65)


# ------------------------------------------------------------------ the cut of the tokens
def test_pieces_are_a_partition_that_the_launch_holds(tmp_path):
    exe = str(tmp_path / "kv_split_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", os.path.join(ROOT, "tests", "host", "kv_split_check.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr


# ------------------------------------------------------------------ refusals of the C ABI
def _cache(**kw):
    c = dict(K_pool=FAKE, V_pool=FAKE, K_scale=FAKE, V_scale=FAKE, act_pool=None, block_table=FAKE, seq_len=FAKE, total_tokens=100,
             P_kv=10, P_act=0, n_act_used=0, block_tokens=16, max_blocks=8, n_kv_heads=8, format=hk.HK_KV_INT8)
    c.update(kw)
    return hk.hk_kv_cache(**c)


def _decode(shape=None, q=FAKE, B=4, lp=None, out=FAKE, ws=FAKE, ws_bytes=1 << 40, **kw):
    shape = shape or hk.make_shape(4096, 32)
    return hk.lib().hk_kv_decode_attn(ctypes.byref(shape), q, B, ctypes.byref(_cache(**kw)), ctypes.byref(lp) if lp else None, out, ws, ws_bytes, None)


def _tree(q=FAKE, k=FAKE, v=FAKE, B=4, T=8, mask=None, stride=0, nodes=None, **kw):
    shape = hk.make_shape(4096, 32)
    return hk.lib().hk_kv_tree_attn(ctypes.byref(shape), q, k, v, B, T, mask, stride, nodes, ctypes.byref(_cache(**kw)), None, FAKE, FAKE, 1 << 40, None)


def _store(k=FAKE, v=FAKE, x=None, B=4, T=8, n_new=None, pick=None, **kw):
    shape = hk.make_shape(1024, 8)
    return hk.lib().hk_kv_store(ctypes.byref(shape), k, v, x, B, T, n_new, pick, ctypes.byref(_cache(**kw)), None)


def _load(K=FAKE, V=FAKE, B=4, off=0, L=8, **kw):
    shape = hk.make_shape(1024, 8)
    return hk.lib().hk_kv_load(ctypes.byref(shape), K, V, B, off, L, ctypes.byref(_cache(**kw)), None)


CACHE_REFUSALS = [
    (dict(format=3), "DTYPE"), (dict(format=-1), "DTYPE"),
    (dict(n_kv_heads=0), "SHAPE"), (dict(n_kv_heads=5), "SHAPE"), (dict(n_kv_heads=-8), "SHAPE"),
    (dict(block_tokens=8), "SHAPE"), (dict(block_tokens=24), "SHAPE"), (dict(block_tokens=2048), "SHAPE"),
    (dict(P_kv=-1), "SHAPE"), (dict(max_blocks=-1), "SHAPE"), (dict(n_act_used=1), "SHAPE"),
    (dict(total_tokens=-1), "SHAPE"), (dict(total_tokens=4 * 8 * 16 + 1), "SHAPE"),
    (dict(max_blocks=1 << 27), "SHAPE"), (dict(P_kv=1 << 30, block_tokens=1024), "SHAPE"),
    (dict(P_act=2, act_pool=FAKE), "SHAPE"),                                             # 8 bits take no ACT blocks
    (dict(block_table=None), "NULL"), (dict(seq_len=None), "NULL"), (dict(K_pool=None), "NULL"), (dict(V_pool=None), "NULL"),
    (dict(K_scale=None), "NULL"), (dict(V_scale=None), "NULL"),
    (dict(K_pool=FAKE + 8), "ALIGN"), (dict(V_scale=FAKE + 4), "ALIGN"), (dict(block_table=FAKE + 2), "ALIGN"), (dict(seq_len=FAKE + 1), "ALIGN"),
]


@pytest.mark.parametrize("call", [_decode, _tree, _store, _load])
@pytest.mark.parametrize("kw,status", CACHE_REFUSALS)
def test_caches_that_every_call_refuses(call, kw, status):
    assert call(**kw) == getattr(hk, "HK_ERR_" + status)


def test_refusals_of_the_attention_calls():
    assert _decode(q=None) == hk.HK_ERR_NULL and _decode(out=None) == hk.HK_ERR_NULL and _decode(ws=None) == hk.HK_ERR_NULL
    assert _decode(q=FAKE + 2) == hk.HK_ERR_ALIGN and _decode(ws=FAKE + 16) == hk.HK_ERR_ALIGN
    assert _decode(hk.make_shape(4096, 31)) == hk.HK_ERR_SHAPE and _decode(hk.make_shape(4096, 32, dtype=2)) == hk.HK_ERR_DTYPE
    assert _decode(B=-1) == hk.HK_ERR_SHAPE and _decode(B=(1 << 20) + 1, total_tokens=0) == hk.HK_ERR_SHAPE
    assert _decode(ws_bytes=64, max_blocks=4096, total_tokens=100000) == hk.HK_ERR_WORKSPACE
    assert _decode(P_kv=0) == hk.HK_ERR_SHAPE                                            # tokens but no block to hold them
    assert _decode(B=0, total_tokens=0) == hk.HK_OK
    # checkpoints: 16 bits, a K/V head of its own for every query head, and the layer
    hybrid = dict(format=hk.HK_KV_16, P_act=2, n_act_used=2, act_pool=FAKE, n_kv_heads=32)
    assert _decode(**hybrid) == hk.HK_ERR_NULL
    assert _decode(lp=hk.hk_layer_params(FAKE, FAKE, FAKE + 2, FAKE, None), **hybrid) == hk.HK_ERR_ALIGN
    assert _decode(**dict(hybrid, n_kv_heads=8)) == hk.HK_ERR_SHAPE
    assert _decode(**dict(hybrid, act_pool=None)) == hk.HK_ERR_NULL
    assert _tree(k=None) == hk.HK_ERR_NULL and _tree(v=None) == hk.HK_ERR_NULL and _tree(q=None) == hk.HK_ERR_NULL
    assert _tree(T=0) == hk.HK_ERR_SHAPE and _tree(T=65) == hk.HK_ERR_SHAPE
    assert _tree(mask=FAKE, stride=7) == hk.HK_ERR_SHAPE and _tree(mask=FAKE, stride=-8) == hk.HK_ERR_SHAPE
    assert _tree(mask=FAKE + 4) == hk.HK_ERR_ALIGN and _tree(nodes=FAKE + 2) == hk.HK_ERR_ALIGN and _tree(v=FAKE + 8) == hk.HK_ERR_ALIGN
    assert _tree(B=0, total_tokens=0) == hk.HK_OK


def test_refusals_of_store_and_load():
    assert _store(k=None) == hk.HK_ERR_NULL and _store(v=None) == hk.HK_ERR_NULL and _store(k=None, v=None) == hk.HK_ERR_NULL
    assert _store(T=-1) == hk.HK_ERR_SHAPE and _store(T=1 << 24) == hk.HK_ERR_SHAPE
    assert _store(k=FAKE + 4) == hk.HK_ERR_ALIGN and _store(pick=FAKE + 1) == hk.HK_ERR_ALIGN and _store(n_new=FAKE + 2) == hk.HK_ERR_ALIGN
    assert _store(x=FAKE + 2) == hk.HK_ERR_ALIGN
    assert _store(T=0) == hk.HK_OK and _store(B=0, total_tokens=0) == hk.HK_OK
    assert _load(K=None) == hk.HK_ERR_NULL and _load(V=None) == hk.HK_ERR_NULL and _load(K=FAKE + 8) == hk.HK_ERR_ALIGN
    assert _load(off=-1) == hk.HK_ERR_SHAPE and _load(L=-1) == hk.HK_ERR_SHAPE and _load(L=1 << 30) == hk.HK_ERR_SHAPE
    # a launch holds fewer than 2^32 threads: 4 requests x 8 heads x 2^18 workgroups of 32 tokens are the last that fit
    assert _load(K=None, L=1 << 23) == hk.HK_ERR_NULL and _load(K=None, L=(1 << 23) + 1) == hk.HK_ERR_SHAPE
    assert _load(L=0) == hk.HK_OK and _load(B=0, total_tokens=0) == hk.HK_OK


def test_workspace_is_known_before_the_pools_are():
    shape, size = hk.make_shape(4096, 32), hk.lib().hk_kv_attn_workspace_bytes
    empty = dict(K_pool=None, V_pool=None, K_scale=None, V_scale=None, block_table=None, seq_len=None)
    ask = lambda B, T, **kw: size(ctypes.byref(shape), B, T, ctypes.byref(_cache(**dict(empty, **kw))))
    assert ask(4, 1) >= 256 and ask(4, 65) == 0 and ask(4, 1, n_kv_heads=3) == 0
    big = dict(max_blocks=4096, total_tokens=60000)
    assert ask(1, 8, **big) >= ask(1, 1, **big) > 256
    hybrid = dict(format=hk.HK_KV_16, P_act=64, n_act_used=64, n_kv_heads=32)
    assert ask(4, 1, **hybrid) >= 2 * 64 * 16 * 4096 * 2


def test_cuts_that_no_launch_holds_are_refused():
    """At most 2^23 workgroups of 256: the pieces of 8 K/V heads (one row), or 2^20 ranges that are merged by 8 (512 rows)."""
    size = hk.lib().hk_kv_attn_workspace_bytes
    shape = hk.make_shape(4096, 32, attn_splits=64)
    ask = lambda B, T: size(ctypes.byref(shape), B, T, ctypes.byref(_cache(max_blocks=1 << 13, total_tokens=B << 17)))
    assert ask(16131, 1) > 0 and ask(16132, 1) == 0        # 16131 * 65 * 8 <= 2^23
    assert ask(1 << 11, 64) > 0 and ask((1 << 11) + 1, 64) == 0


def test_struct_layout():
    assert ctypes.sizeof(hk.hk_kv_cache) == 7 * 8 + 8 + 7 * 4 + 4


# ------------------------------------------------------------------ refusals of the binding
def _tensors(dtype=torch.int8):
    pool = torch.zeros(3, 2, 16, 64, dtype=dtype)
    scale = None if dtype in (torch.float16, torch.bfloat16) else torch.zeros(3, 2, 16)
    return pool, torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), scale


def test_binding_refuses_what_does_not_fit():
    pool, table, lens, scale = _tensors()
    make = hk.make_kv_cache
    with pytest.raises(TypeError):                         # there is no CPU path
        make(pool, pool, table, lens, 16, scale, scale)
    with pytest.raises(TypeError):
        make(pool.float(), pool.float(), table, lens, 16)
    for bad in (lambda: make(pool, pool[:2], table, lens, 16, scale, scale), lambda: make(pool, pool, table, lens, 32, scale, scale),
                lambda: make(pool, pool, table, lens[:1], 16, scale, scale), lambda: make(pool, pool, table[0], lens, 16, scale, scale),
                lambda: make(pool, pool, table, lens, 16), lambda: make(pool, pool, table, lens, 16, scale),
                lambda: make(pool, pool, table, lens, 16, scale[:2], scale),
                lambda: make(pool.half(), pool.half(), table, lens, 16, scale, scale),
                lambda: make(pool.half(), pool.half(), table, lens, 16, act_pool=torch.zeros(2, 8, 128).half())):
        with pytest.raises(ValueError):
            bad()


class _Handle(hk.KvCache):
    """A handle as make_kv_cache builds it, without a GPU behind it."""

    def __init__(self, B=2, Hkv=2, dh=64, form=hk.HK_KV_INT8, el=torch.int8, n_act_used=0):
        self.struct = hk.hk_kv_cache(n_kv_heads=Hkv, format=form, block_tokens=16, max_blocks=4, n_act_used=n_act_used)
        self.ref, self.tensors, self.device, self.index, self.pool_dtype = ctypes.byref(self.struct), (), torch.device("cuda:0"), 0, el
        self.B, self.n_kv_heads, self.head_dim, self.d_act, self.shapes = B, Hkv, dh, None, {}


class _Gpu:
    """What the binding looks at of a GPU tensor."""

    def __init__(self, *shape, dtype=torch.float16, device=0, contiguous=True, is_cuda=True):
        self.shape, self.dtype, self.is_cuda, self._contiguous = torch.Size(shape), dtype, is_cuda, contiguous
        self.device = torch.device("cuda:%d" % device)

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self.device.index

    def is_contiguous(self):
        return self._contiguous

    def data_ptr(self):
        return FAKE


def test_calls_of_the_binding_refuse_what_does_not_fit():
    c, z = _Handle(), _Gpu
    i32 = lambda *s: _Gpu(*s, dtype=torch.int32)
    rows, q = z(2, 3, 2, 64), z(2, 3, 4, 64)
    class side:
        device = torch.device("cuda:1")
    for bad in (lambda: hk.kv_store(c, rows, z(1, 3, 2, 64)), lambda: hk.kv_store(c, z(2, 3, 1, 64), z(2, 3, 1, 64)),
                lambda: hk.kv_store(c, z(1, 3, 2, 64), z(1, 3, 2, 64)), lambda: hk.kv_store(c, rows, rows, n_new=i32(3)),
                lambda: hk.kv_store(c, rows, rows, pick=i32(2, 2)), lambda: hk.kv_store(c, rows, rows, x=z(2, 3, 64)),
                lambda: hk.kv_store(c, z(2, 2, 64), z(2, 2, 64)), lambda: hk.kv_store(c, rows, z(2, 3, 2, 64, device=1)),
                lambda: hk.kv_store(c, rows, rows, stream=side), lambda: hk.kv_store(c, rows, z(2, 3, 2, 64, contiguous=False)),
                lambda: hk.kv_load(c, 5, K_out=z(2, 2, 5, 64)), lambda: hk.kv_load(c, 5, K_out=z(2, 2, 5, 64), V_out=z(2, 2, 5, 64), stream=side),
                lambda: hk.kv_decode_attn(q, c), lambda: hk.kv_decode_attn(z(3, 4, 64), c), lambda: hk.kv_decode_attn(z(2, 4, 128), c),
                lambda: hk.kv_decode_attn(z(2, 4, 64, device=1), c), lambda: hk.kv_decode_attn(z(2, 2, 64), _Handle(n_act_used=1)),
                lambda: hk.kv_decode_attn(z(2, 4, 64), c, workspace=z(4096, dtype=torch.uint8, device=1)),
                lambda: hk.kv_decode_attn(z(2, 4, 64), c, layer_params=(z(100),) * 4),
                lambda: hk.kv_decode_attn(z(2, 4, 64), c, layer_params=(z(256, device=1),) * 4),
                lambda: hk.kv_tree_attn(z(2, 4, 64), rows, rows, c), lambda: hk.kv_tree_attn(q, z(2, 2, 2, 64), rows, c),
                lambda: hk.kv_tree_attn(q, rows, z(2, 3, 4, 64), c), lambda: hk.kv_tree_attn(q, rows, rows, c, mask=z(2, dtype=torch.int64)),
                lambda: hk.kv_tree_attn(q, rows, rows, c, mask=z(3, 3, dtype=torch.int64)), lambda: hk.kv_tree_attn(q, rows, rows, c, n_nodes=i32(3))):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: hk.kv_decode_attn(z(2, 4, 64, dtype=torch.float32), c), lambda: hk.kv_store(c, z(2, 3, 2, 64, dtype=torch.float32), rows),
                lambda: hk.kv_decode_attn(z(2, 4, 64, dtype=torch.bfloat16), _Handle(form=hk.HK_KV_16, el=torch.float16)),
                lambda: hk.kv_store(c, rows, z(2, 3, 2, 64, dtype=torch.bfloat16)), lambda: hk.kv_store(c, rows, rows, n_new=z(2, dtype=torch.int64)),
                lambda: hk.kv_tree_attn(q, rows, rows, c, mask=i32(3)), lambda: hk.kv_store(c, rows, z(2, 3, 2, 64, is_cuda=False)),
                lambda: hk.kv_load(c, 4, dtype=torch.float32), lambda: hk.kv_store(c, torch.zeros(2, 3, 2, 64).half(), rows)):
        with pytest.raises(TypeError):
            bad()
