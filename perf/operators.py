"""The operators of the 8-bit and 16-bit paged K/V cache, as cases that can be timed and compared.

  store   kv_store: K/V rows of new tokens quantised into the blocks of a paged cache, then read back with kv_load
  load    kv_load: the rows of a quantised cache as contiguous 16-bit K/V
  decode  kv_decode_attn: one query token a request over the cache
  tree    kv_tree_attn: a tree of drafted tokens a request over the cache and over each node's ancestors

``own`` selects the framework's calls; otherwise ``run`` computes the same in elementary torch operations in 32 bits.  Inputs
have the scales of the repository's recipe (``synth.py``).  What a serving loop keeps between steps (the cache's handle, output
buffers, workspaces, the prepared layer) is kept in the state.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
MOST = {"int8": 127.0, "e4m3": 448.0}
LEAST_SCALE = 2.0 ** -100


def listed():
    return [
        # The smallest write: one token of four requests of the smallest layer.
        _case("store_one", "store", (12, 12, 64), "f16", "int8", B=4, L_min=200, L_max=256, T=1),
        # Prompts of different lengths enter a cache of a layer with shared K/V heads.
        _case("store_prompt", "store", (32, 8, 128), "bf16", "e4m3", B=8, L_min=1024, L_max=2048, T=2048),
        # A batch of requests leaves the quantised cache for calls that want 16 bits.
        _case("load_batch", "load", (32, 32, 128), "f16", "int8", B=32, L_min=512, L_max=1024),
        # Three long documents, read back.
        _case("load_long", "load", (32, 8, 128), "bf16", "e4m3", B=3, L_min=20001, L_max=30001, block=64),
        # One request: the latency of a chat.
        _case("decode_one", "decode", (32, 8, 128), "f16", "int8", B=1, L_min=1999, L_max=1999),
        # An ordinary batch of the 6.7B-shaped layer.
        _case("decode_batch", "decode", (32, 32, 128), "f16", "int8", B=32, L_min=512, L_max=1024),
        # The largest cache: the benchmark's batch and context, every token cached.
        _case("decode_largest", "decode", (72, 72, 128), "bf16", "e4m3", B=64, L_min=2048, L_max=4096),
        # Long contexts with eight query heads on a K/V head, 16-bit cache.
        _case("decode_long_shared", "decode", (64, 8, 128), "bf16", "16", B=4, L_min=16384, L_max=32768, block=64),
        # The smallest verification: eight drafted tokens of one short request.
        _case("tree_tiny", "tree", (12, 12, 64), "f16", "16", B=1, L_min=200, L_max=256, T=8),
        # Half of the blocks checkpoints, whose regeneration serves all drafted tokens.
        _case("tree_hybrid", "tree", (32, 32, 128), "f16", "16", B=8, L_min=512, L_max=1024, T=24, act_share=0.5),
        # A full tree of 64 nodes over long contexts, eight query heads on a K/V head: 512 query rows per K/V head.
        _case("tree_shared", "tree", (64, 8, 128), "bf16", "int8", B=16, L_min=4096, L_max=8192, T=64),
        # Odd sizes: tiles of tokens, of nodes and of rows that do not come out even.
        _case("tree_odd", "tree", (40, 40, 128), "f16", "e4m3", B=7, L_min=383, L_max=1148, T=33),
    ]


def _case(name, path, heads, dtype, form, B, L_min, L_max, T=1, block=16, act_share=0.0, pick=False):
    return {"name": name, "path": path, "heads": heads[0], "kv_heads": heads[1], "dh": heads[2], "dtype": dtype, "form": form,
            "B": B, "L_min": L_min, "L_max": L_max, "T": T, "block": block, "act_share": act_share, "pick": pick}


def _log_uniform(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    path = rng.choice(["store", "load", "decode", "decode", "tree", "tree"])
    heads = rng.choice([(12, 12, 64), (32, 32, 128), (40, 40, 128), (72, 72, 128), (32, 8, 128), (64, 8, 128), (16, 2, 64), (28, 4, 128)])
    B = _log_uniform(rng, 1, 128)
    # at most the K/V elements of the largest listed cache, and for a tree at most the products of the largest listed one
    most = min(32768, 64 * 1400 * 72 // (B * heads[1]))
    T = 1
    if path == "tree":
        T = rng.randint(2, 64)
        most = min(most, 16 * 4096 * 64 * 64 // (B * T * heads[0]))
    L = _log_uniform(rng, 16, max(17, most))
    form = rng.choice(["int8", "e4m3"] if path in ("store", "load") else ["int8", "e4m3", "16"])
    dtype, act_share = rng.choice(["f16", "bf16"]), 0.0
    d = heads[0] * heads[2]
    if path == "tree" and form == "16" and heads[0] == heads[1] and B * L * d * d <= 8 * 768 * 4096 ** 2 and rng.random() < 0.7:
        # checkpoints: fp16, in which a regenerated row keeps 11 bits; no more of them than in the listed case
        dtype, act_share = "f16", round(0.5 * rng.random(), 2)
    pick = path == "store" and rng.random() < 0.5
    if path == "store":
        T = rng.choice([1, min(L, rng.randint(2, 64)), L])
    case = _case("", path, heads, dtype, form, B=B, L_min=max(1, L // 2), L_max=L, T=T, block=rng.choice([16, 16, 32, 64, 128]),
                 act_share=act_share, pick=pick and T <= 64)
    del case["name"]
    return case


# ----------------------------------------------------------------------------------------------------------- inputs
def _lengths(case):
    """Request lengths: part of the case (not of the seed), so that the work is the same for every seed."""
    return np.random.default_rng(case["L_max"] * 1009 + case["B"]).integers(case["L_min"], case["L_max"] + 1, case["B"])


def _nodes(case):
    """Nodes of every request's tree, or its tokens to store."""
    if case["path"] == "store":
        lens = _lengths(case)
        return lens if case["T"] >= case["L_max"] else np.minimum(lens, case["T"])
    return np.random.default_rng(case["T"] * 31 + case["B"]).integers((case["T"] + 1) // 2, case["T"] + 1, case["B"])


def _blocks(case):
    """Blocks of every request, KV blocks and ACT blocks in all."""
    counts = (_lengths(case) + case["block"] - 1) // case["block"]
    act = round(case["act_share"] * int(counts.sum()))
    return counts, int(counts.sum()) - act, act


def _table(case, rng):
    counts, n_kv, n_act = _blocks(case)
    entries = rng.permutation(np.concatenate([rng.permutation(n_kv), ~rng.permutation(n_act)])).astype(np.int32)
    table = np.zeros((case["B"], int(counts.max())), np.int32)
    at = 0
    for b, n in enumerate(counts):
        table[b, :n] = entries[at:at + n]
        at += n
    return torch.from_numpy(table).cuda()


def _masks(B, T, rng):
    """Ancestors of every node and the node itself, as bits: node i hangs on the context (a root) or on an earlier node."""
    mask = np.zeros((B, T), np.uint64)
    for b in range(B):
        for i in range(T):
            parent = int(rng.integers(-1, i)) if i else -1
            mask[b, i] = np.uint64(1 << i) | (mask[b, parent] if parent >= 0 else np.uint64(0))
    return torch.from_numpy(mask.view(np.int64)).cuda()


def _quantise(x, form):
    """Codes and scales of rows x[..., dh], in the cache's definition (fp32)."""
    x = x.float()
    most = torch.full((), MOST[form], device=x.device)     # a tensor: by a plain number torch multiplies with its reciprocal
    scale = (x.abs().amax(-1, keepdim=True) / most).clamp_min(LEAST_SCALE)
    y = x / scale
    code = y.round().clamp(-127, 127).to(torch.int8) if form == "int8" else y.to(torch.float8_e4m3fn)
    return code, scale.squeeze(-1)


def prepare(case, seed):
    el, form, path = DTYPES[case["dtype"]], case["form"], case["path"]
    H, Hkv, dh, B, T, bt = case["heads"], case["kv_heads"], case["dh"], case["B"], case["T"], case["block"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    d, std = H * dh, 0.02 * (H * dh) ** 0.5

    def normal(*shape, std=1.0, mean=0.0):
        return torch.empty(shape, dtype=el, device="cuda").normal_(mean, std, generator=gen)

    lens = _lengths(case)
    _, n_kv, n_act = _blocks(case)
    s = {"path": path, "form": form, "block": bt, "H": H, "T": T, "n_act": n_act, "scales": (None, None), "act": None, "layer": None}
    pools = []
    for _ in range(2):
        rows = normal(n_kv + 1, Hkv, bt, dh, std=std)      # the last block is free
        pools.append((rows, None) if form == "16" else _quantise(rows, form))
        del rows
    s["pools"] = tuple(p[0] for p in pools)
    if form != "16":
        s["scales"] = tuple(p[1] for p in pools)
    s["table"], s["lens"] = _table(case, rng), torch.from_numpy(lens.astype(np.int32)).cuda()
    s["L"] = int(lens.max())
    if n_act:
        s["act"] = normal(n_act, bt, d)
        s["layer"] = (normal(d, std=0.02, mean=1.0), normal(d, std=0.02), normal(2 * d, d, std=0.02), normal(2 * d, std=0.01))
    if path in ("store", "tree"):
        s["k"], s["v"] = normal(B, T, Hkv, dh, std=std), normal(B, T, Hkv, dh, std=std)
        s["nodes"] = torch.from_numpy(_nodes(case).astype(np.int32)).cuda()
    if path == "store":
        # the path through the draft that was accepted: the node of each token
        path_nodes = np.sort(rng.integers(0, T, (B, T)), 1).astype(np.int32) if case["pick"] else None
        s["pick"] = None if path_nodes is None else torch.from_numpy(path_nodes).cuda()
    if path in ("store", "load"):
        s["K"], s["V"] = (torch.zeros(B, Hkv, s["L"], dh, dtype=el, device="cuda") for _ in range(2))
    if path == "decode":
        s["q"] = normal(B, H, dh, std=std)
        s["out"] = torch.zeros_like(s["q"])
    if path == "tree":
        s["q"] = normal(B, T, H, dh, std=std)
        s["out"] = torch.zeros_like(s["q"])
        s["mask"] = _masks(B, T, rng)
    if own:
        _handles(s, int(lens.sum()))
    return s


def _handles(s, total):
    """What a program that serves with the framework sets up once: the cache's handle, the workspace, the prepared layer."""
    from paper_2501_01792_amd import binding as hk
    s["cache"] = hk.make_kv_cache(*s["pools"], s["table"], s["lens"], s["block"], *s["scales"], act_pool=s["act"], total_tokens=total)
    if s["path"] in ("decode", "tree"):
        s["ws"] = hk.new_workspace(hk.kv_attn_workspace_bytes(s["q"], s["cache"]))
    if s["layer"] is not None:
        s["layer"] = s["layer"] + (hk.prepare_layer(*s["layer"], s["H"]),)


# -------------------------------------------------------------------------------------------------------- one pass
def run(s):
    if own:
        return _run_own(s)
    if s["path"] == "store":
        _store(s)
    if s["path"] in ("store", "load"):
        return _load(s)
    return _attend(s)


def _run_own(s):
    from paper_2501_01792_amd import binding as hk
    path = s["path"]
    if path == "store":
        hk.kv_store(s["cache"], s["k"], s["v"], n_new=s["nodes"], pick=s["pick"])
    if path in ("store", "load"):
        return hk.kv_load(s["cache"], s["L"], K_out=s["K"], V_out=s["V"])
    if path == "decode":
        return hk.kv_decode_attn(s["q"], s["cache"], out=s["out"], workspace=s["ws"])
    return hk.kv_tree_attn(s["q"], s["k"], s["v"], s["cache"], mask=s["mask"], n_nodes=s["nodes"], layer_params=s["layer"],
                           out=s["out"], workspace=s["ws"])


def _store(s):
    B, T = s["k"].shape[:2]
    i = torch.arange(T, device="cuda")
    new = i < s["nodes"][:, None]
    source = s["pick"].long() if s["pick"] is not None else i.expand(B, T)
    token = ((s["lens"] - s["nodes"])[:, None] + i).clamp_max(s["table"].shape[1] * s["block"] - 1)
    free = s["pools"][0].shape[0] - 1                      # the block that takes what is behind a request's new tokens
    block = torch.where(new, s["table"].gather(1, token // s["block"]).long(), free)
    row = token % s["block"]
    for x, pool, scale in zip((s["k"], s["v"]), s["pools"], s["scales"]):
        code, sc = _quantise(x.gather(1, source[..., None, None].expand(x.shape)), s["form"])
        pool.view(torch.int8)[block, :, row] = code.view(torch.int8)
        scale[block, :, row] = sc


def _rows(s, which):
    """K or V of every request as [B, Hkv, blocks * block, dh] in fp32."""
    pool, scale = s["pools"][which].float(), s["scales"][which]
    if scale is not None:
        pool = pool * scale[..., None]
    at = s["table"].long()
    if s["act"] is not None:
        pool = torch.cat([pool, _regenerate(s, which)])
        at = torch.where(at < 0, pool.shape[0] - s["n_act"] + ~at, at)
    rows = pool[at].transpose(1, 2)
    return rows.reshape(rows.shape[0], rows.shape[1], -1, rows.shape[-1])


def _regenerate(s, which):
    ln_w, ln_b, W, b = (t.float() for t in s["layer"][:4])
    d, x = ln_w.shape[0], s["act"].float()
    x = x - x.mean(-1, keepdim=True)
    x = x / (x.square().mean(-1, keepdim=True) + 1e-5).sqrt() * ln_w + ln_b
    y = x.reshape(-1, d) @ W[which * d:(which + 1) * d].t().contiguous() + b[which * d:(which + 1) * d]
    return y.reshape(s["n_act"], s["block"], s["H"], -1).transpose(1, 2)


def _load(s):
    here = (torch.arange(s["L"], device="cuda") < s["lens"][:, None])[:, None, :, None]
    return tuple(torch.where(here, _rows(s, w)[:, :, :s["L"]].to(old.dtype), old) for w, old in ((0, s["K"]), (1, s["V"])))


def _attend(s):
    tree = s["path"] == "tree"
    q = s["q"] if tree else s["q"][:, None]
    B, T, H, dh = q.shape
    K, V = _rows(s, 0), _rows(s, 1)
    Hkv, L = K.shape[1], K.shape[2]
    seen = (torch.arange(L, device="cuda") < s["lens"][:, None])[:, None].expand(B, T, L)
    if tree:
        node = torch.arange(T, device="cuda")
        K = torch.cat([K, s["k"].float().transpose(1, 2)], 2)
        V = torch.cat([V, s["v"].float().transpose(1, 2)], 2)
        bits = (s["mask"][..., None] >> node & 1).bool() & (node < s["nodes"][:, None])[:, None]
        seen = torch.cat([seen, bits], 2)
    q = q.float().reshape(B, T, Hkv, H // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dh)
    score = (q * dh ** -0.5) @ K.transpose(2, 3).contiguous()
    seen = seen[:, None, None].expand(B, Hkv, H // Hkv, T, seen.shape[-1]).reshape(B, Hkv, -1, seen.shape[-1])
    score = score.masked_fill_(~seen, -torch.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp_(score.sub_(torch.where(top > -torch.inf, top, torch.zeros_like(top))))
    total = p.sum(-1, keepdim=True)
    out = (p @ V) / torch.where(total > 0, total, torch.ones_like(total))
    out = out.reshape(B, Hkv, H // Hkv, T, dh).permute(0, 3, 1, 2, 4).reshape(B, T, H, dh).to(s["out"].dtype)
    if not tree:
        return out[:, 0]
    return torch.where((torch.arange(T, device="cuda") < s["nodes"][:, None])[..., None, None], out, s["out"])


# ------------------------------------------------------------------------------------------------- exact values, work
def exact(case, seed):
    """Request by request in 64 bits, from the definitions."""
    s = prepare(case, seed)
    Q, form, bt = MOST.get(s["form"]), s["form"], s["block"]
    lens, table = s["lens"].tolist(), s["table"].tolist()
    f64 = torch.float64

    def value(which, e):
        if e < 0:
            return regenerated[which][~e]
        rows = s["pools"][which][e].to(f64)
        return rows if s["scales"][which] is None else rows * s["scales"][which][e].to(f64)[..., None]

    def context(which, b):
        n = lens[b]
        return torch.cat([value(which, e) for e in table[b][:(n + bt - 1) // bt]], 1)[:, :n]

    def requantised(x):
        scale = torch.maximum(x.abs().amax(-1, keepdim=True) / Q, torch.tensor(LEAST_SCALE, dtype=f64, device="cuda"))
        y = x / scale
        if form == "int8":
            return torch.round(y) * scale
        # e4m3: three bits behind the leading one, spacing no finer than 2^-9
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
        return torch.round(y / step) * step * scale

    if s["act"] is not None:
        ln_w, ln_b, W, bias = (t.to(f64) for t in s["layer"][:4])
        x = s["act"].to(f64)
        var, mean = torch.var_mean(x, -1, unbiased=False, keepdim=True)
        y = ((x - mean) / torch.sqrt(var + 1e-5) * ln_w + ln_b) @ W.t() + bias
        both = y.reshape(s["n_act"], bt, 2, s["H"], -1).permute(2, 0, 3, 1, 4)
        regenerated = (both[0], both[1])
    if s["path"] in ("store", "load"):
        outs = []
        for which, old in ((0, s["K"]), (1, s["V"])):
            out = old.to(f64)
            for b, n in enumerate(lens):
                out[b, :, :n] = context(which, b)
                if s["path"] == "store":
                    new = int(s["nodes"][b])
                    at = s["pick"][b, :new].long() if s["pick"] is not None else slice(0, new)
                    out[b, :, n - new:n] = requantised((s["k"], s["v"])[which][b, at].to(f64)).transpose(0, 1)
            outs.append(out)
        return tuple(outs)
    g, dh = s["H"] // case["kv_heads"], case["dh"]
    out = s["out"].to(f64)
    for b, n in enumerate(lens):
        K, V = context(0, b), context(1, b)
        nodes = int(s["nodes"][b]) if s["path"] == "tree" else 1
        q = s["q"][b, :nodes].to(f64) if s["path"] == "tree" else s["q"][b:b + 1].to(f64)
        seen = torch.ones(nodes, K.shape[1], dtype=torch.bool, device="cuda")
        if s["path"] == "tree":
            K = torch.cat([K, s["k"][b, :nodes].to(f64).transpose(0, 1)], 1)
            V = torch.cat([V, s["v"][b, :nodes].to(f64).transpose(0, 1)], 1)
            bits = [[bool(m >> j & 1) for j in range(nodes)] for m in s["mask"][b, :nodes].tolist()]
            seen = torch.cat([seen, torch.tensor(bits, dtype=torch.bool, device="cuda")], 1)
        for h in range(case["kv_heads"]):
            score = q[:, h * g:(h + 1) * g].reshape(-1, dh) @ K[h].t() / math.sqrt(dh)
            score = score.masked_fill(~seen.repeat_interleave(g, 0), -torch.inf)
            o = (torch.softmax(score, -1) @ V[h]).reshape(nodes, g, dh)
            if s["path"] == "tree":
                out[b, :nodes, h * g:(h + 1) * g] = o
            else:
                out[b, h * g:(h + 1) * g] = o[0]
    return out


def work(case):
    """Bytes: what is read once and what is written once.  Flops: the products of scores and of the weighted sum, and of the
    regeneration where blocks are checkpoints."""
    H, Hkv, dh, path = case["heads"], case["kv_heads"], case["dh"], case["path"]
    tokens, bt = int(_lengths(case).sum()), case["block"]
    row = 4 * dh if case["form"] == "16" else 2 * (dh + 4)             # K and V of one token and head, as they are held
    wide = 4 * dh                                                      # the same in 16 bits
    if path == "load":
        return {"bytes": tokens * Hkv * (row + wide), "flops": 2 * tokens * Hkv * dh}
    if path == "store":
        new = int(_nodes(case).sum())
        return {"bytes": (new + tokens) * Hkv * (row + wide), "flops": 2 * (new + tokens) * Hkv * dh}
    rows, square = case["B"], 0
    if path == "tree":
        nodes = _nodes(case)
        rows, square = int(nodes.sum()), int((nodes * nodes).sum())
        pairs = int((_lengths(case) * nodes).sum()) + square
    else:
        pairs = tokens
    _, n_kv, n_act = _blocks(case)
    held = min(tokens, n_act * bt)
    nbytes = (tokens - held) * Hkv * row + 4 * rows * H * dh + (wide * rows * Hkv if path == "tree" else 0)
    flops = 4 * pairs * H * dh
    if n_act:
        d = H * dh
        nbytes += 2 * held * d + 4 * d * d
        flops += 4 * held * d * d
    return {"bytes": nbytes, "flops": flops}
