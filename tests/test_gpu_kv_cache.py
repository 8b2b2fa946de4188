"""The paged K/V cache in 16 bits, int8 and e4m3 on the GPU, through the binding, against its oracle in 64 bits: rows written and
read back, attention of one token and of drafted trees, and the calls as a serving loop strings them together."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import hybridkv_oracle as ho
from oracle import kv_oracle as ko
from paper_2501_01792_amd import binding as hk

pytestmark = pytest.mark.gpu
EL = {"f16": torch.float16, "bf16": torch.bfloat16}
HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}         # a rounding to the type is off by so much of the value at most
POOL = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def f64(t):
    return t.double().cpu().numpy()


class Cache:
    """A cache with random content (stale rows and spare blocks among it) on the GPU, and the same on the host."""

    def __init__(self, seed, form, dtype, lens, Hkv, dh, bt, max_blocks=None, std=1.0, spare=2, total=None):
        rng = np.random.default_rng(seed)
        self.form, self.dtype, self.bt, self.Hkv, self.dh = form, dtype, bt, Hkv, dh
        counts = [(n + bt - 1) // bt for n in lens]
        max_blocks = max_blocks or max(max(counts), 1)
        P = sum(counts) + spare
        ids = rng.permutation(P)
        self.table = np.full((len(lens), max_blocks), 0x7fffffff, np.int32)      # never read behind a request's blocks
        at = 0
        for r, c in enumerate(counts):
            self.table[r, :c] = ids[at:at + c]
            at += c
        gen = torch.Generator().manual_seed(seed)
        rows = [(torch.randn(P, Hkv, bt, dh, generator=gen) * std).to(EL[dtype]) for _ in range(2)]
        self.lens = np.asarray(lens, np.int32)
        if form == "16":
            self.pools, self.scales = [r.cuda() for r in rows], [None, None]
        else:
            both = [ko.quantise(r.float().numpy(), form) for r in rows]
            self.pools = [torch.from_numpy(c.view(np.int8)).cuda().view(POOL[form]) for c, _ in both]
            self.scales = [torch.from_numpy(s).cuda() for _, s in both]
        self.dtable, self.dlens = torch.from_numpy(self.table).cuda(), torch.from_numpy(self.lens).cuda()
        self.handle = hk.make_kv_cache(*self.pools, self.dtable, self.dlens, bt, *self.scales,
                                       total_tokens=int(np.maximum(self.lens, 0).sum()) if total is None else total)

    def context(self, which, r, n=None):
        pool = self.pools[which]
        pool = pool.double().cpu().numpy() if self.form == "16" else \
            pool.view(torch.int8).cpu().numpy().view(np.int8 if self.form == "int8" else np.uint8)
        scale = None if self.form == "16" else self.scales[which].cpu().numpy()
        return ko.context(pool, scale, self.table[r], int(self.lens[r]) if n is None else n, self.form)


def normal(seed, *shape, dtype="f16", std=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * std).to(EL[dtype]).cuda()


def within(name, got, ref, size, most, peak, dtype, half, n):
    """|got - ref| held to what the roundings allow, `half` being half a step of the type that the weights are rounded to.
      * The result: half a step of its type; fp16's smallest numbers, 2^-25.
      * The weights: half a step each, a part of sum p |v| (`size`).  A weight below fp16's normal numbers is off by 2^-25
        against a largest weight between a half and one: n tokens, 2^-24 of the largest p |v| (`peak`) each.
      * The scores: dh <= 128 products summed in fp32 are off by 128 2^-24 of sum |q k| scale (`most`); eight more roundings of
        the size of the score (fp16 queries made from bf16 ones among them).  A change of all scores by x changes the weights
        and their sum by a part x each, so 2 x.
      * Sums of n weights and products in fp32, the pieces' factors and exp2: (n + 64) 2^-24."""
    bound = half * size + HALF_STEP[dtype] * np.abs(ref) + 2.0 ** -25 + n * 2.0 ** -24 * peak \
        + (2 * 136 * 2.0 ** -24 * (1 + most) + (n + 64) * 2.0 ** -24) * size
    off = np.abs(got - ref)
    print("%s: max_abs=%.3e, %.2f of the bound" % (name, off.max(initial=0), (off / bound).max(initial=0)), flush=True)
    assert (off <= bound).all(), "%s: %.3e over" % (name, (off - bound).max())


# ------------------------------------------------------------------ rows written, rows read back
STORES = [
    # form, dtype, Hkv, dh, bt, lens, n_new (None: T), T
    ("int8", "f16", 2, 64, 16, [1, 17, 40], None, 1),
    ("int8", "bf16", 3, 128, 32, [40, 33, 64, 5], [33, 0, 40, 5], 40),
    ("e4m3", "f16", 1, 128, 16, [100], [77], 90),
    ("e4m3", "bf16", 8, 64, 64, [7, 130, 64], [9, -1, 1000], 19),       # more than the request has, negative, more than T
    ("16", "f16", 5, 64, 16, [20, 1], None, 3),
    ("16", "bf16", 4, 128, 1024, [1030, 3], [1029, 3], 1030),
]


@pytest.mark.parametrize("form,dtype,Hkv,dh,bt,lens,n_new,T", STORES)
@pytest.mark.parametrize("pick", [False, True])
def test_store_and_load(form, dtype, Hkv, dh, bt, lens, n_new, T, pick):
    B = len(lens)
    c = Cache(1, form, dtype, lens, Hkv, dh, bt)
    gen = torch.Generator().manual_seed(2)
    k, v = (torch.randn(B, T, Hkv, dh, generator=gen) * 10.0 ** (torch.rand(B, T, Hkv, 1, generator=gen) * 7 - 4) for _ in range(2))
    k[0, 0, 0] = 0                                         # a row of zeros, an infinity, a NaN, the type's smallest and largest
    k, v = k.to(EL[dtype]), v.to(EL[dtype])
    v[0, 0, 0, 3], v[-1, -1, -1, -1] = float("inf"), float("nan")
    if T > 2:
        k[-1, 1], k[-1, 2, 0, 1] = torch.finfo(EL[dtype]).smallest_normal / 4, torch.finfo(EL[dtype]).max
        v[-1, 1, :, 5:] = 0
    before = [p.clone() for p in c.pools], [s if s is None else s.clone() for s in c.scales]
    picks = np.random.default_rng(3).integers(-2, T + 2, (B, T)).astype(np.int32) if pick else None
    n = [T if n_new is None else min(max(n_new[r], 0), T) for r in range(B)]
    hk.kv_store(c.handle, k.cuda(), v.cuda(), n_new=None if n_new is None else torch.tensor(n_new, dtype=torch.int32).cuda(),
                pick=None if picks is None else torch.from_numpy(picks).cuda())
    torch.cuda.synchronize()
    for x, pool, scale, was, was_scale in ((k, c.pools[0], c.scales[0], before[0][0], before[1][0]), (v, c.pools[1], c.scales[1], before[0][1], before[1][1])):
        want, want_scale = was.cpu().clone(), None if scale is None else was_scale.cpu().clone()
        for r in range(B):
            for i in range(n[r]):
                t, src = lens[r] - n[r] + i, i if picks is None else int(picks[r, i])
                if t < 0 or not 0 <= src < T:
                    continue
                e = int(c.table[r, t // bt])
                if form == "16":
                    want[e, :, t % bt] = x[r, src]
                else:
                    code, sc = ko.quantise(x[r, src].float().numpy(), form)
                    want.view(torch.int8)[e, :, t % bt] = torch.from_numpy(code.view(np.int8))
                    want_scale[e, :, t % bt] = torch.from_numpy(sc)
        raw = torch.int16 if form == "16" else torch.int8
        got, want = pool.cpu().view(raw), want.view(raw)
        assert torch.equal(got, want), "%d of %d codes differ" % (int((got != want).sum()), got.numel())
        if scale is not None:
            assert torch.equal(torch.nan_to_num(scale.cpu(), nan=-1.0), torch.nan_to_num(want_scale, nan=-1.0))
    for off, L_cap in ((0, max(lens)), (0, 1), (5, 70), (max(lens), 4)):
        K_out, V_out = (torch.full((B, Hkv, L_cap, dh), 7.0, dtype=EL[dtype], device="cuda") for _ in range(2))
        hk.kv_load(c.handle, L_cap, tok_off=off, K_out=K_out, V_out=V_out)
        torch.cuda.synchronize()
        for which, out in ((0, K_out), (1, V_out)):
            for r in range(B):
                here = max(0, min(L_cap, lens[r] - off))
                ref = c.context(which, r)[:, off:off + here]
                # scale * code in fp32 (2^-24), rounded once (half a step); fp16's smallest numbers: half of 2^-24
                got, fine = f64(out[r, :, :here]), np.isfinite(ref)
                assert (np.isnan(got) == np.isnan(ref)).all() and (got[~fine & ~np.isnan(ref)] == ref[~fine & ~np.isnan(ref)]).all()
                assert (np.abs(got - ref)[fine] <= (HALF_STEP[dtype] + 2.0 ** -23) * np.abs(ref[fine]) + 2.0 ** -25).all()
                assert (out[r, :, here:] == 7.0).all()


def test_load_in_a_type_of_the_callers_choice():
    c = Cache(4, "int8", "bf16", [20], 2, 64, 16)
    K, V = hk.kv_load(c.handle, 24, dtype=torch.bfloat16)
    assert K.dtype == torch.bfloat16 and K.shape == (1, 2, 24, 64) and (K[:, :, 20:] == 0).all()
    assert np.abs(f64(V[0, :, :20]) - c.context(1, 0)).max() <= 2.0 ** -8 * 5
    assert hk.kv_load(c.handle, 3)[0].dtype == torch.float16


def test_store_into_checkpoint_blocks():
    """The rows of new tokens whose block is an ACT block are layer inputs; KV blocks take K and V."""
    B, T, H, dh, bt, d = 2, 20, 2, 64, 16, 128
    K, V, act = (torch.zeros(3, H, bt, dh).half().cuda(), torch.zeros(3, H, bt, dh).half().cuda(), torch.zeros(2, bt, d).half().cuda())
    table, lens = torch.tensor([[2, ~1, 99], [~0, 0, 99]], dtype=torch.int32).cuda(), torch.tensor([25, 18], dtype=torch.int32).cuda()
    cache = hk.make_kv_cache(K, V, table, lens, bt, act_pool=act)
    k, v, x = normal(1, B, T, H, dh), normal(2, B, T, H, dh), normal(3, B, T, d)
    for given in (None, x):
        hk.kv_store(cache, k, v, x=given, n_new=torch.tensor([20, 18], dtype=torch.int32).cuda())
        assert torch.equal(K[2, :, 5:], k[0, :11].transpose(0, 1)) and torch.equal(V[0, :, :2], v[1, 16:18].transpose(0, 1))
        assert (act == 0).all() if given is None else torch.equal(act[1, :9], x[0, 11:20]) and torch.equal(act[0], x[1, :16])
    assert (K[1] == 0).all() and (K[2, :, :5] == 0).all() and (act[1, 9:] == 0).all()
    out = torch.full((B, H, 25, dh), 7.0).half().cuda()
    hk.kv_load(cache, 25, K_out=out, V_out=out.clone())
    assert torch.equal(out[0, :, 5:16], k[0, :11].transpose(0, 1)) and (out[0, :, 16:] == 7).all() and (out[1, :, :16] == 7).all()


# ------------------------------------------------------------------ one token
DECODES = [
    # dh, H, Hkv, bt, lens
    (64, 12, 12, 16, [1, 0, 31, 32, 33, 200]),
    (128, 8, 1, 32, [129, 4, 1000, 0]),
    (128, 40, 40, 16, [383]),
    (64, 16, 2, 128, [2000, 5]),
    (128, 34, 2, 64, [257, 640]),                          # 17 heads on a K/V head: two tiles of rows
]


def check_attention(name, c, q, k, v, mask, nodes, out, untouched=None, scale=None):
    B, T, H, dh = q.shape
    scale = dh ** -0.5 if scale is None else scale
    got = f64(out)
    for r in range(B):
        n = T if nodes is None else min(max(int(nodes[r]), 0), T)
        seen = np.zeros((n, n), bool)
        for i in range(n):
            for j in range(n):
                m = (1 << i + 1) - 1 if mask is None else int(mask[r, i] if mask.dim() == 2 else mask[i])
                seen[i, j] = m >> j & 1
        K, V = c.context(0, r), c.context(1, r)
        ref, size, most, peak = ko.tree_attention(f64(q[r, :n]), None if k is None else f64(k[r, :n]), None if k is None else f64(v[r, :n]), K, V, seen, scale)
        # over an 8-bit cache the weights are fp16; those of the nodes are of the rows' type
        half = HALF_STEP[c.dtype if c.form == "16" or k is not None else "f16"]
        within("%s[%d]" % (name, r), got[r, :n], ref, size, most, peak, c.dtype, half, K.shape[1] + n)
        if untouched is not None:
            assert (got[r, n:] == untouched).all()


@pytest.mark.parametrize("dh,H,Hkv,bt,lens", DECODES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("splits", [0, 1, 7])
def test_decode(dh, H, Hkv, bt, lens, dtype, form, splits):
    c = Cache(dh + H, form, dtype, lens, Hkv, dh, bt)
    q = normal(5, len(lens), H, dh, dtype=dtype, std=1.5)
    ws = hk.new_workspace(hk.kv_attn_workspace_bytes(q, c.handle, splits))
    ws.fill_(0xff)                                         # NaN wherever scratch is read before it is written
    out = hk.kv_decode_attn(q, c.handle, workspace=ws, attn_splits=splits)
    check_attention("decode", c, q[:, None], None, None, None, None, out[:, None])
    assert all((out[r] == 0).all() for r, n in enumerate(lens) if n == 0)


def test_decode_with_a_total_that_is_only_a_bound_and_lengths_beyond_the_table():
    c = Cache(8, "e4m3", "f16", [70, 300, 1], 2, 64, 16, total=None)
    q = normal(6, 3, 4, 64)
    want = f64(hk.kv_decode_attn(q, c.handle))
    loose = hk.make_kv_cache(*c.pools, c.dtable, c.dlens, 16, *c.scales)
    got = f64(hk.kv_decode_attn(q, loose))
    assert np.abs(got - want).max() <= 2.0 ** -10 * np.abs(want).max()
    # a length that the table's row has no room for is the room; a negative one is nothing
    c.dtable[0] = c.dtable[1]
    c.dlens.copy_(torch.tensor([1 << 30, 304, -5], dtype=torch.int32))
    out = hk.kv_decode_attn(q[1:2].expand(3, 4, 64).contiguous(), loose)
    assert torch.equal(out[0], out[1]) and (out[2] == 0).all()


def test_sixteen_bits_agree_with_the_hybrid_caches_own_attention():
    lens, H, dh, bt = [300, 17, 64], 12, 64, 16
    c = Cache(9, "16", "f16", lens, H, dh, bt)
    q = normal(7, 3, H, dh)
    cu = torch.tensor([0, 300, 317, 381], dtype=torch.int64).cuda()
    table = torch.where(c.dtable == 0x7fffffff, torch.zeros_like(c.dtable), c.dtable)
    want = hk.paged_decode_attn(q, *c.pools, None, table, c.dlens, bt, None, cu_tokens=cu, total_tokens=381)
    got = hk.kv_decode_attn(q, c.handle)
    # both are within two half steps (weights and result) of the exact result, whose rows are sums of |v| < 4
    assert (got.float() - want.float()).abs().max() <= 4 * 2.0 ** -11 * 4


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_scales_of_every_size(form, dtype):
    """Tokens whose V scales lie far apart, rows of zeros among them, and bf16 queries beyond fp16's range: a weight keeps its
    bits, and the denominator counts the tokens whose V is nothing."""
    lens, H, dh, bt = [90, 64], 4, 64, 16
    c = Cache(10, form, dtype, lens, 2, dh, bt)
    gen = torch.Generator().manual_seed(11)
    for r, e in enumerate(c.scales[1].flatten(0, 1)):
        e.mul_(10.0 ** (torch.rand(bt, generator=gen) * 10 - 7).cuda())
    c.scales[1][:, :, 3] = 0.0
    c.scales[1][:, :, 5] = 2.0 ** -100
    c.pools[1].view(torch.int8)[:, :, 3] = 0
    c.pools[1].view(torch.int8)[:, :, 5] = 0
    q = normal(12, 2, H, dh, dtype=dtype)
    if dtype == "bf16":
        q[1, 0] *= 2.0 ** 20                               # the scale of the keys takes it back
        q[1, 1] *= 2.0 ** -40
        c.scales[0][:, 0] *= 2.0 ** -18
    out = hk.kv_decode_attn(q, c.handle)
    check_attention("scales", c, q[:, None], None, None, None, None, out[:, None])


@pytest.mark.parametrize("form", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,power", [("f16", -12), ("f16", 10), ("bf16", -40), ("bf16", 40)])
@pytest.mark.parametrize("T", [5, 30])
def test_a_tree_keeps_the_bits_of_small_and_large_v(form, dtype, power, T):
    """V of cache and nodes far from one: the nodes' rows have no scale that stands beside the tokens' ones."""
    lens, H, Hkv, dh, bt = [300, 70, 0], 4, 2, 64, 16
    c = Cache(100, form, dtype, lens, Hkv, dh, bt)
    q, k, v = normal(101, 3, T, H, dh, dtype=dtype), normal(102, 3, T, Hkv, dh, dtype=dtype), normal(103, 3, T, Hkv, dh, dtype=dtype)
    for splits in (0, 3):
        c.scales[1].mul_(2.0 ** power)
        out = hk.kv_tree_attn(q, k, v * 2.0 ** power, c.handle, attn_splits=splits)
        if dtype == "bf16":                                # exact powers of two: held to the tolerance at V of size one
            c.scales[1].mul_(2.0 ** -power)
            check_attention("power", c, q, k, v, None, None, out.double() * 2.0 ** -power)
        else:
            check_attention("power", c, q, k, v * 2.0 ** power, None, None, out)
            c.scales[1].mul_(2.0 ** -power)


def test_many_short_requests_and_one_long_one():
    """More requests than a wavefront has lanes, most of them short or empty, in every form that cuts their tokens."""
    rng = np.random.default_rng(104)
    lens = [int(n) for n in rng.integers(0, 40, 150)]
    lens[3], lens[64], lens[130], lens[149] = 0, 5000, 0, 700
    for form, T, H in (("int8", 1, 8), ("16", 3, 8), ("e4m3", 9, 16), ("int8", 17, 40)):
        c = Cache(105, form, "f16", lens, 2, 64, 32)
        q, k, v = normal(106, 150, T, H, 64), normal(107, 150, T, 2, 64), normal(108, 150, T, 2, 64)
        nodes = rng.integers(0, T + 1, 150).astype(np.int32)
        for splits in (0, 1, 2):
            if T == 1:
                check_attention("ragged", c, q, None, None, None, None, hk.kv_decode_attn(q[:, 0].contiguous(), c.handle, attn_splits=splits)[:, None])
            else:
                out = torch.full_like(q, 7.0)
                hk.kv_tree_attn(q, k, v, c.handle, n_nodes=torch.from_numpy(nodes).cuda(), out=out, attn_splits=splits)
                check_attention("ragged", c, q, k, v, None, nodes, out, untouched=7.0)


# ------------------------------------------------------------------ trees
def random_masks(seed, B, T, kind):
    rng = np.random.default_rng(seed)
    if kind == "tree":
        return torch.stack([hk.tree_mask([-1] + [int(rng.integers(-1, i)) for i in range(1, T)]) for _ in range(B)])
    if kind == "one":
        return hk.tree_mask([-1] + [int(rng.integers(-1, i)) for i in range(1, T)])
    m = rng.integers(-2 ** 63, 2 ** 63, (B, T))            # any pattern, bits of nodes that there are not among it
    m[:, 0] = 0                                            # a node that sees no node
    return torch.from_numpy(m)


TREES = [
    # dh, H, Hkv, bt, T, lens, nodes, kind of mask
    (64, 4, 4, 16, 1, [5, 0], None, None),
    (64, 12, 12, 16, 8, [200], None, "tree"),
    (128, 4, 4, 32, 17, [0, 40, 100], [17, 0, 9], "any"),
    (64, 16, 2, 16, 33, [64, 0, 1], [33, 1, 20], "one"),
    (128, 8, 1, 64, 64, [130, 300], [64, 50], "tree"),     # 512 rows on a K/V head
    (64, 6, 2, 16, 64, [31, 500], None, None),             # a chain; 3 heads on a K/V head
    (128, 5, 5, 16, 48, [700], [47], "any"),
]


@pytest.mark.parametrize("dh,H,Hkv,bt,T,lens,nodes,kind", TREES)
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form", ["16", "int8", "e4m3"])
@pytest.mark.parametrize("splits", [0, 1, 3])
def test_tree(dh, H, Hkv, bt, T, lens, nodes, kind, dtype, form, splits):
    B = len(lens)
    c = Cache(dh + T, form, dtype, lens, Hkv, dh, bt)
    q, k, v = normal(13, B, T, H, dh, dtype=dtype), normal(14, B, T, Hkv, dh, dtype=dtype), normal(15, B, T, Hkv, dh, dtype=dtype)
    mask = None if kind is None else random_masks(16, B, T, kind)
    out = torch.full_like(q, 7.0)
    ws = hk.new_workspace(hk.kv_attn_workspace_bytes(q, c.handle, splits))
    ws.fill_(0xff)
    hk.kv_tree_attn(q, k, v, c.handle, mask=None if mask is None else mask.cuda(), out=out, workspace=ws, attn_splits=splits,
                    n_nodes=None if nodes is None else torch.tensor(nodes, dtype=torch.int32).cuda())
    check_attention("tree", c, q, k, v, mask, nodes, out, untouched=7.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("form", ["16", "e4m3"])
@pytest.mark.parametrize("dh", [64, 128])
def test_what_a_node_does_not_see_has_no_influence(dtype, form, dh):
    """NaN and infinities in rows behind the cached tokens, in nodes that a node does not see and behind the last node."""
    lens, H, Hkv, bt, T = [21, 0], 4, 2, 16, 40
    c = Cache(17, form, dtype, lens, Hkv, dh, bt)
    q, k, v = normal(18, 2, T, H, dh, dtype=dtype), normal(19, 2, T, Hkv, dh, dtype=dtype), normal(20, 2, T, Hkv, dh, dtype=dtype)
    nodes = torch.tensor([39, 40], dtype=torch.int32).cuda()
    mask = random_masks(21, 2, T, "any")
    wild = 1 << 3 | 1 << 7 | 1 << 36 | 1 << 39
    mask &= ~wild
    mask[0, 5] |= 1 << 7                                   # one node sees the NaN, two an infinity
    mask[1, 6] |= 1 << 36
    mask[1, 8] |= 1 << 3
    clean = hk.kv_tree_attn(q, k, v, c.handle, mask=mask.cuda(), n_nodes=nodes)
    for x in (k, v):
        x[:, 3], x[:, 7], x[:, 39] = float("inf"), float("nan"), float("nan")
    v[:, 36, :, 1], v[:, 36, :, 2] = float("inf"), float("-inf")
    if form == "16":
        for p in c.pools:
            p[c.table[0, 1], :, 5:] = float("nan")
    else:
        for p, s in zip(c.pools, c.scales):
            p.view(torch.int8)[c.table[0, 1], :, 5:] = 0x7f
            s[c.table[0, 1], :, 5:] = float("nan")
    got = hk.kv_tree_attn(q, k, v, c.handle, mask=mask.cuda(), n_nodes=nodes)
    hit = torch.zeros(2, T, dtype=torch.bool)
    hit[0, 5] = hit[1, 6] = hit[1, 8] = True
    assert torch.equal(got[~hit], clean[~hit]) and torch.isfinite(got[~hit]).all()
    assert torch.isnan(got[0, 5]).all() and not torch.isfinite(got[1, 8]).any()
    a = got[1, 6].float()
    assert (a[:, 1] == float("inf")).all() and (a[:, 2] == float("-inf")).all()
    rest = [e for e in range(dh) if e not in (1, 2)]
    assert torch.equal(got[1, 6][:, rest], clean[1, 6][:, rest])


def test_hybrid_blocks_serve_a_tree():
    """ACT blocks are regenerated once for all nodes: against the oracle's regenerated rows; and one token against the hybrid
    cache's own attention on the same blocks."""
    B, T, H, dh, bt, d = 2, 9, 4, 64, 16, 256
    lens = [70, 33]
    K, V, act = normal(23, 5, H, bt, dh), normal(24, 5, H, bt, dh), normal(25, 4, bt, d)
    table = np.array([[4, ~1, 0, ~3, 2], [~0, ~2, 1, 77, 77]], np.int32)
    lp = (normal(26, d, std=0.02) + 1, normal(27, d, std=0.02), normal(28, 2 * d, d, std=0.02), normal(29, 2 * d, std=0.01))
    cache = hk.make_kv_cache(K, V, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), bt, act_pool=act)
    q, k, v = normal(30, B, T, H, dh), normal(31, B, T, H, dh), normal(32, B, T, H, dh)
    mask = random_masks(33, B, T, "tree")
    h = [t.cpu().numpy() for t in lp]
    rk, rv = ho.regen_kv(act.cpu().numpy().astype(np.float64), h[0], h[1], h[2], h[3], H)
    for params in (lp, lp + (hk.prepare_layer(*lp, H),)):
        out = hk.kv_tree_attn(q, k, v, cache, mask=mask.cuda(), layer_params=params)
        one = hk.kv_decode_attn(q[:, 0].contiguous(), cache, layer_params=params)
        for r, n in enumerate(lens):
            pick = lambda pool, regen: np.concatenate([f64(pool[e]) if e >= 0 else regen[~e] for e in table[r, :(n + bt - 1) // bt]], 1)[:, :n]
            Kc, Vc = pick(K, rk), pick(V, rv)
            seen = np.array([[int(mask[r, i]) >> j & 1 for j in range(T)] for i in range(T)], bool)
            for got, nodes, sees in ((out[r], T, seen), (one[r][None], 1, None)):
                ref = ko.tree_attention(f64(q[r, :nodes]), f64(k[r]) if sees is not None else None, f64(v[r]), Kc, Vc, sees, dh ** -0.5)[0]
                # the tolerance of the step that regenerates, which the paged calls are held to elsewhere
                assert np.abs(f64(got) - ref).max() <= 2e-2 and np.linalg.norm(f64(got) - ref) <= 5e-3 * np.linalg.norm(ref)
        cu = torch.tensor([0, 70, 103], dtype=torch.int64).cuda()
        want = hk.paged_decode_attn(q[:, 0].contiguous(), K, V, act, cache.tensors[5], cache.tensors[6], bt, params, cu_tokens=cu, total_tokens=103)
        assert (one.float() - want.float()).abs().max() <= 4 * 2.0 ** -11 * 4


def test_rows_beyond_32_bits():
    """Blocks at the far end of pools of more than 2^32 bytes: rows written there are read and attended over."""
    Hkv, dh, bt, P = 8, 128, 64, 66000                     # 4.3e9 codes in each pool
    pools = [torch.zeros(P, Hkv, bt, dh, dtype=torch.int8, device="cuda") for _ in range(2)]
    scales = [torch.zeros(P, Hkv, bt, device="cuda") for _ in range(2)]
    table = torch.tensor([[P - 1, 3, P - 2]], dtype=torch.int32).cuda()
    lens = torch.tensor([150], dtype=torch.int32).cuda()
    cache = hk.make_kv_cache(*pools, table, lens, bt, *scales)
    k, v, q = normal(34, 1, 150, Hkv, dh), normal(35, 1, 150, Hkv, dh), normal(36, 1, 16, dh)
    hk.kv_store(cache, k, v)
    K, V = hk.kv_load(cache, 150)
    for x, out in ((k, K), (v, V)):
        code, sc = ko.quantise(x[0].transpose(0, 1).float().cpu().numpy(), "int8")
        assert (np.abs(f64(out[0]) - ko.dequantise(code, sc, "int8")) <= 2.0 ** -11 * 5).all()
    small = Cache(37, "int8", "f16", [150], Hkv, dh, bt)
    for far, near in zip(pools + scales, small.pools + small.scales):
        for i, e in enumerate((P - 1, 3, P - 2)):
            near[small.table[0, i]] = far[e]
    assert torch.equal(hk.kv_decode_attn(q, cache), hk.kv_decode_attn(q, small.handle))


# ------------------------------------------------------------------ streams, graphs, a serving loop
def test_side_stream_and_repeated_calls_give_the_same_bits():
    c = Cache(38, "e4m3", "bf16", [900, 3, 411], 2, 128, 16)
    q, k, v = (normal(39 + i, 3, 20, h, 128, dtype="bf16") for i, h in enumerate((8, 2, 2)))
    want = hk.kv_tree_attn(q, k, v, c.handle)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = [hk.kv_tree_attn(q, k, v, c.handle, stream=side) for _ in range(4)]
    K, V = hk.kv_load(c.handle, 900, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(o, want) for o in outs)
    K2, V2 = hk.kv_load(c.handle, 900)
    assert torch.equal(K, K2) and torch.equal(V, V2)


def test_two_graphs_that_share_a_workspace():
    """A graph that stores and verifies and one that decodes, captured once; between the replays lengths, tables and rows change
    and other work runs."""
    H, Hkv, dh, bt, T = 8, 2, 64, 16, 5
    c = Cache(40, "int8", "f16", [40, 700], Hkv, dh, bt, max_blocks=64, spare=90, total=2 * 64 * 16)
    c.dtable[:] = torch.arange(128, dtype=torch.int32).view(2, 64)
    c.table = c.dtable.cpu().numpy()
    q, k, v, q1 = normal(41, 2, T, H, dh), normal(42, 2, T, Hkv, dh), normal(43, 2, T, Hkv, dh), normal(44, 2, H, dh)
    n_new, nodes, mask = (torch.tensor(x).cuda() for x in (np.array([2, 1], np.int32), np.array([5, 3], np.int32), random_masks(45, 2, T, "tree").numpy()))
    out, out1 = torch.zeros_like(q), torch.zeros_like(q1)
    ws = hk.new_workspace(max(hk.kv_attn_workspace_bytes(q, c.handle), hk.kv_attn_workspace_bytes(q1, c.handle)))

    def verify():
        hk.kv_store(c.handle, k, v, n_new=n_new)
        hk.kv_tree_attn(q, k, v, c.handle, mask=mask, n_nodes=nodes, out=out, workspace=ws)

    def decode():
        hk.kv_decode_attn(q1, c.handle, out=out1, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graphs = []
    with torch.cuda.stream(side):
        verify(), decode()
        for call in (verify, decode):
            graphs.append(torch.cuda.CUDAGraph())
            with torch.cuda.graph(graphs[-1], stream=side):
                call()
    torch.cuda.current_stream().wait_stream(side)
    for step, lens in enumerate(([43, 701], [100, 16], [1, 1000], [640, 0])):
        c.dlens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = np.asarray(lens, np.int32)
        for i, x in enumerate((q, k, v, q1)):
            x.copy_(normal(50 + 10 * step + i, *x.shape))
        torch.randn(1 << 20, device="cuda").sum()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        got, got1 = out.clone(), out1.clone()
        check_attention("replay %d" % step, c, q, k, v, mask.cpu(), nodes.cpu(), got)
        check_attention("replay %d" % step, c, q1[:, None], None, None, None, None, got1[:, None])
        ws.fill_(0xff)
        verify(), decode()
        assert torch.equal(out[0], got[0]) and torch.equal(out[1, :3], got[1, :3]) and torch.equal(out1, got1)


@pytest.mark.parametrize("T,H", [(9, 8), (24, 8)])         # 36 and 96 rows on a K/V head: ranges of one tile of rows and of two
def test_a_graph_of_ranges_follows_the_lengths(T, H):
    """The cut of many rows is found on the device: one capture serves lengths and trees of every size."""
    c = Cache(110, "e4m3", "bf16", [40, 700, 5], 2, 128, 16, max_blocks=64, spare=200, total=3 * 64 * 16)
    c.dtable[:] = torch.arange(192, dtype=torch.int32).view(3, 64)
    c.table = c.dtable.cpu().numpy()
    q, k, v = (normal(111 + i, 3, T, h, 128, dtype="bf16") for i, h in enumerate((H, 2, 2)))
    nodes, out = torch.full((3,), T, dtype=torch.int32).cuda(), torch.zeros_like(q)
    ws = hk.new_workspace(hk.kv_attn_workspace_bytes(q, c.handle))
    call = lambda: hk.kv_tree_attn(q, k, v, c.handle, n_nodes=nodes, out=out, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.current_stream().wait_stream(side)
    for lens, n in (([1000, 1, 33], [T, 1, T]), ([0, 0, 1024], [0, T, T - 1]), ([0, 0, 0], [0, 0, 0]), ([512, 640, 31], [T, T, T])):
        c.lens = np.asarray(lens, np.int32)
        c.dlens.copy_(torch.from_numpy(c.lens))
        nodes.copy_(torch.tensor(n, dtype=torch.int32))
        out.fill_(7.0)
        torch.randn(1 << 20, device="cuda").sum()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        check_attention("ranges", c, q, k, v, None, n, got, untouched=7.0)
        ws.fill_(0xff)
        out.fill_(7.0)
        call()
        assert torch.equal(out, got)


@pytest.mark.parametrize("form", ["int8", "e4m3", "16"])
def test_speculative_decoding_over_a_quantised_cache(form):
    """The calls of a serving loop, in turn: prompts of different lengths are stored; each step drafts a tree whose Q, K, V come
    from hk_qkv_current, verifies it, stores an accepted path and decodes the next token over what is cached then.  Every
    result is held to attention over the rows as the cache holds them."""
    d, H, bt, T, B = 256, 4, 16, 7, 3
    dh = d // H
    prompts, max_blocks = [30, 1, 64], 12
    lp = (normal(60, d, std=0.02) + 1, normal(61, d, std=0.02), normal(62, 2 * d, d, std=0.05), normal(63, 2 * d, std=0.01))
    Wq, bq = normal(64, d, d, std=0.05), normal(65, d, std=0.01)
    c = Cache(66, form, "f16", [0] * B, H, dh, bt, max_blocks=max_blocks, spare=B * max_blocks, total=B * max_blocks * bt)
    c.dtable.copy_(torch.randperm(B * max_blocks, generator=torch.Generator().manual_seed(67)).view(B, max_blocks))
    c.table = c.dtable.cpu().numpy()
    held = [np.zeros((2, H, 0, dh)) for _ in range(B)]      # what the cache should hold, exactly as its format does

    def project(x):
        n = x.shape[0] * x.shape[1]
        k, v = (torch.empty(n, H, 1, dh, dtype=torch.float16, device="cuda") for _ in range(2))
        q = hk.qkv_current(x.reshape(n, d), *lp, Wq, bq, H, K_dst=k, V_dst=v)
        return (t.view(x.shape[0], x.shape[1], H, dh) for t in (q, k, v))

    def as_held(row):
        return f64(row) if form == "16" else ko.dequantise(*ko.quantise(row.float().cpu().numpy(), form), form)

    def set_lens(lens):
        c.lens = np.asarray(lens, np.int32)
        c.dlens.copy_(torch.from_numpy(c.lens))

    def store(k, v, n_new, pick=None):
        set_lens([int(n) + m for n, m in zip(c.lens, n_new)])
        hk.kv_store(c.handle, k, v, n_new=torch.tensor(n_new, dtype=torch.int32).cuda(), pick=None if pick is None else torch.tensor(pick, dtype=torch.int32).cuda())
        for r in range(B):
            at = list(range(n_new[r])) if pick is None else pick[r][:n_new[r]]
            new = np.stack([np.stack([as_held(x[r, i]) for i in at], 1) for x in (k, v)]) if at else np.zeros((2, H, 0, dh))
            held[r] = np.concatenate([held[r], new], 2)
            for which in (0, 1):
                assert np.abs(c.context(which, r) - held[r][which]).max(initial=0) <= 1e-12

    _, k, v = project(normal(68, B, 64, d))
    store(k, v, prompts)
    rng = np.random.default_rng(69)
    for step in range(4):
        q, k, v = project(normal(70 + step, B, T, d))
        parents = [-1, 0, 0, 1, 1, 3, 2]
        mask = hk.tree_mask(parents)
        out = hk.kv_tree_attn(q, k, v, c.handle, mask=mask.cuda())
        check_attention("verify %d" % step, c, q, k, v, mask, None, out)
        paths = ([0, 1, 3, 5], [0, 2, 6], [0])
        accepted = [paths[int(rng.integers(3))] for _ in range(B)]
        store(k, v, [len(p) for p in accepted], [p + [0] * (T - len(p)) for p in accepted])
        q, k, v = project(normal(80 + step, B, 1, d))
        store(k, v, [1] * B)
        one = hk.kv_decode_attn(q[:, 0].contiguous(), c.handle)
        check_attention("decode %d" % step, c, q, None, None, None, None, one[:, None])


def test_refusals_touch_nothing():
    c = Cache(90, "int8", "f16", [20], 2, 64, 16)
    q = normal(91, 1, 4, 64)
    out = torch.full_like(q, 7.0)
    with pytest.raises(hk.HybridKVError):
        hk.kv_decode_attn(normal(92, 1, 3, 64), c.handle, out=torch.empty(1, 3, 64, dtype=torch.float16, device="cuda"))   # 3 heads on 2
    with pytest.raises(hk.HybridKVError):
        hk.kv_decode_attn(q, c.handle, out=out, workspace=torch.empty(100, dtype=torch.uint8, device="cuda"), attn_splits=3)
    with pytest.raises(hk.HybridKVError):
        hk.kv_tree_attn(normal(93, 1, 65, 4, 64), *(normal(94, 1, 65, 2, 64),) * 2, c.handle)
    with pytest.raises(ValueError):
        hk.kv_decode_attn(q.transpose(1, 2).contiguous().transpose(1, 2), c.handle, out=out)
    with pytest.raises(TypeError):
        hk.kv_tree_attn(normal(95, 1, 2, 4, 64), *(normal(96, 1, 2, 2, 64),) * 2, c.handle, mask=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        hk.kv_decode_attn(q, c.handle, workspace=torch.empty(4096, dtype=torch.uint8))
    torch.cuda.synchronize()
    assert (out == 7.0).all()
