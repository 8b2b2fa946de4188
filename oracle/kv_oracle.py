"""TEST INFRASTRUCTURE -- NOT PART OF THE PRODUCT PATH.

The paged K/V cache in 16 bits, int8 and e4m3 and the attention over it, stated plainly in numpy: rows are quantised one by one
from the definition, requests, heads and nodes are handled one after the other in 64 bits.  It imports nothing from the GPU
package.

Pins (tests/test_kv_cache_host.py): hand-computed codes, the half step that a rounding may be off by, the e4m3 values listed by
their bits, and attention over one token, over equal scores and over nothing.
"""
import numpy as np

Q = {"int8": 127.0, "e4m3": 448.0}
LEAST_SCALE = np.float32(2.0 ** -100)


def e4m3_values():
    """The value of each of the 256 codes (sign, 4 exponent bits with bias 7, 3 mantissa bits; S.1111.111 is NaN)."""
    out = np.empty(256)
    for code in range(256):
        e, f = code >> 3 & 15, code & 7
        v = (1 + f / 8) * 2.0 ** (e - 7) if e else f / 8 * 2.0 ** -6
        out[code] = np.nan if code & 127 == 127 else -v if code & 128 else v
    return out


_E4M3 = e4m3_values()
_POSITIVE = _E4M3[:127]                                    # increasing


def e4m3_code(y):
    """Nearest code of |y| <= 464, ties to the even mantissa."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    lo = hi - 1
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantise(x, form):
    """Rows x[..., dh] (16-bit values in any float type) -> codes (int8, or uint8 bits of e4m3) and fp32 scales [...]."""
    x = np.asarray(x, np.float32)
    top = np.abs(x).max(-1)
    fine = np.isfinite(x).all(-1)
    scale = np.maximum(np.where(fine, top, 0).astype(np.float32) / np.float32(Q[form]), LEAST_SCALE).astype(np.float32)
    y = np.where(fine[..., None], x, np.float32(0)) / scale[..., None]
    code = np.clip(np.rint(y), -127, 127).astype(np.int8) if form == "int8" else e4m3_code(y.astype(np.float64))
    return code, np.where(fine, scale, np.float32(np.nan))


def dequantise(code, scale, form):
    v = code.astype(np.float64) if form == "int8" else _E4M3[code]
    return v * scale.astype(np.float64)[..., None]


def context(pool, scale, table_row, n, form):
    """Rows [Hkv, n, dh] of a request in 64 bits (pools: 16-bit values as floats, or codes)."""
    bt = pool.shape[2]
    rows = [pool[e].astype(np.float64) if form == "16" else dequantise(pool[e], scale[e], form) for e in table_row[:(n + bt - 1) // bt]]
    if not rows:
        return np.zeros((pool.shape[1], 0, pool.shape[3]))
    return np.concatenate(rows, 1)[:, :n]


def attend(q, K, V, seen, scale):
    """q[dh] over the rows K, V[n, dh] that `seen` names, in 64 bits: out; for tolerances sum p |v|, the largest sum |q k| scale
    and the largest p |v|."""
    dh = q.shape[-1]
    if not seen.any():
        return np.zeros(dh), np.zeros(dh), 0.0, 0.0
    K, V = K[seen], V[seen]
    s = K @ q * scale
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ V, p @ np.abs(V), float((np.abs(K) @ np.abs(q)).max() * scale), float((p[:, None] * np.abs(V)).max())


def tree_attention(q, k, v, K, V, mask, scale):
    """One request: q[n, H, dh], nodes' rows k, v[n, Hkv, dh] (n nodes), context K, V[Hkv, L, dh], mask[n, n] booleans ->
    out[n, H, dh], and as attend() the sums p |v| and the largest of the two others over all rows."""
    n, H, dh = q.shape
    Hkv, L = K.shape[:2]
    out, size, most, peak = np.zeros((n, H, dh)), np.zeros((n, H, dh)), 0.0, 0.0
    for h in range(H):
        hk = h // (H // Hkv)
        keys = np.concatenate([K[hk], k[:, hk]]) if n and k is not None else K[hk]
        vals = np.concatenate([V[hk], v[:, hk]]) if n and k is not None else V[hk]
        for i in range(n):
            seen = np.concatenate([np.ones(L, bool), mask[i]]) if k is not None else np.ones(L, bool)
            out[i, h], size[i, h], a, b = attend(q[i, h].astype(np.float64), keys, vals, seen, scale)
            most, peak = max(most, a), max(peak, b)
    return out, size, most, peak
