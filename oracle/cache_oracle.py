"""fp64 oracle of rotary positions, the paged cache and attention over it, sequence by sequence from the definitions.

Arrays are numpy; a cache is a dict with k_pages, v_pages [n_pages, H_kv, page_size, d] (float64 values, or e4m3 codes as
uint8 with k_scales, v_scales [n_pages, H_kv, page_size]) and block_table [B, max_pages].
"""
import numpy as np

from . import fp8_oracle


def rope(x, inv_freq, positions, rot_dim, interleaved, amplitude=1.0, transposed=False):
    """x [B,H,N,d] float64 with the first rot_dim elements of each row turned by positions [B,N] * inv_freq radians."""
    y = np.array(x, dtype=np.float64)
    phi = np.asarray(positions, dtype=np.float64)[:, None, :, None] * np.asarray(inv_freq, dtype=np.float64)
    c, s = amplitude * np.cos(phi), amplitude * np.sin(phi) * (-1.0 if transposed else 1.0)
    i = np.arange(rot_dim // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot_dim // 2)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., a] * s + x[..., b] * c
    return y


def frequencies(rot_dim, base, scaling="plain", factor=1.0, trained_len=0.0):
    """(inv_freq, amplitude) by the published formulas; `scaling`: plain, linear, ntk or by_parts."""
    i = np.arange(rot_dim // 2, dtype=np.float64)
    if scaling == "ntk":
        base = base * factor ** (rot_dim / (rot_dim - 2.0))
    f = np.exp(-(2.0 * i / rot_dim) * np.log(base))
    if scaling == "linear":
        f = f / factor
    if scaling == "by_parts":
        ramp = np.clip((trained_len / (2.0 * np.pi / f) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        return (1.0 - ramp) * f / factor + ramp * f, 0.1 * np.log(factor) + 1.0
    return f, 1.0


def quantise_rows(x):
    """Codes (uint8) and scales of x [..., d], a row of d at a time, in fp32 as the cache defines them."""
    x = np.asarray(x, dtype=np.float32)
    with np.errstate(invalid="ignore", over="ignore"):
        a = np.where(np.isfinite(x), np.abs(x), np.float32(0)).max(axis=-1)
        a = np.where(a > 0, np.maximum(a, np.float32(2.0 ** -100)), np.float32(0)).astype(np.float32)
        safe = np.where(a > 0, a, np.float32(448))
        z = (x * (np.float32(448) / safe)[..., None]).astype(np.float32)
        codes = fp8_oracle.e4m3_encode(np.where(np.isnan(z), np.float32(0), np.clip(z, -448, 448)))
    return np.where(np.isnan(z), np.uint8(0x7F), codes).astype(np.uint8), (safe / np.float32(448)).astype(np.float32)


def place(cache, b, p):
    """(page, slot) of place p of sequence b, or None"""
    n_pages, _, page_size, _ = cache["k_pages"].shape
    table = cache["block_table"]
    if p // page_size >= table.shape[1]:
        return None
    page = int(table[b, p // page_size])
    return (page, p % page_size) if 0 <= page < n_pages else None


def values(cache, name, places):
    """Rows [n, H_kv, d] of K or V (`name`) in (page, slot) places, float64"""
    pages = cache[name + "_pages"]
    at = np.array(places, dtype=np.int64).reshape(-1, 2)
    rows = pages[at[:, 0], :, at[:, 1]]
    if pages.dtype != np.uint8:
        return rows.astype(np.float64)
    return fp8_oracle.e4m3_decode(rows) * cache[name + "_scales"][at[:, 0], :, at[:, 1]].astype(np.float64)[..., None]


def attend(q, cache, lens, counts, tree, scale):
    """For every row with a count: {(b, h, t): (o [d], lse, K seen [n, d], V seen [n, d])}; q [B,H,T,d] float64, tree: bool
    [B, T, T] or None."""
    B, H, T, _ = q.shape
    group = H // cache["k_pages"].shape[1]
    out = {}
    for b in range(B):
        n, count = max(int(lens[b]), 0), min(int(counts[b]), T)
        places = [place(cache, b, p) for p in range(n)]
        old = [p for p in places if p is not None]
        new = [place(cache, b, n + u) for u in range(count)]
        K0, V0 = (values(cache, x, old) for x in ("k", "v"))
        for t in range(count):
            seen = [new[u] for u in range(count) if new[u] is not None and (u <= t if tree is None else tree[b, t, u])]
            K1, V1 = (values(cache, x, seen) for x in ("k", "v"))
            for h in range(H):
                g = h // group
                K, V = (np.concatenate((y0[:, g], y1[:, g])) for y0, y1 in ((K0, K1), (V0, V1)))
                if len(K) == 0:
                    out[b, h, t] = (np.zeros(q.shape[-1]), -np.inf, K, V)
                    continue
                s = scale * (K @ q[b, h, t])
                m = s.max()
                p = np.exp(s - m)
                out[b, h, t] = (p @ V / p.sum(), m + np.log(p.sum()), K, V)
    return out
