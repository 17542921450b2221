"""The quantised key-value cache in numpy, from its definition (tests only): pages unpacked, rows quantised, attention in 64 bits."""
import numpy as np

PHILOX_M, PHILOX_W = (0xD2511F53, 0xCD9E8D57), (0x9E3779B9, 0xBB67AE85)


def padded(dim):
    return 64 if dim <= 64 else 128 if dim <= 128 else 256


def head_sections(pages, heads, dim, page, bits):
    """pages uint32 [n][words] -> symbols of keys and values [n][heads][page][padded], norms [n][heads][page] of both."""
    p, n = padded(dim), pages.shape[0]
    rk, rv = (p * (b + 1) // 32 for b in bits)
    w = pages.reshape(n, heads, page * (rk + rv + 2))
    cut = np.cumsum([page * rk, page * rv, page])
    ck, cv, nk, nv = np.split(w, cut, axis=2)

    def symbols(c, b):
        s = (c[..., None] >> (np.arange(0, 32, b + 1, dtype=np.uint32))) & np.uint32((1 << (b + 1)) - 1)
        return s.reshape(n, heads, page, p)

    return symbols(ck, bits[0]), symbols(cv, bits[1]), nk.copy().view(np.float32), nv.copy().view(np.float32)


def values_of(symbols, norms, levels):
    """The fp32 product of a signed level with its row's norm, in 64 bits (exact: 11 times 24 bits)."""
    lv = np.asarray(levels, np.float64)
    return lv[symbols >> 1] * np.where(symbols & 1, -1.0, 1.0) * norms.astype(np.float64)[..., None]


def philox_words(seed, c0, c1, c2, c3):
    c0, c1, c2, c3 = (np.broadcast_to(np.asarray(c, np.uint64), np.broadcast(c0, c1, c2, c3).shape).copy() for c in (c0, c1, c2, c3))
    k0, k1, mask = seed & 0xFFFFFFFF, seed >> 32, np.uint64(0xFFFFFFFF)
    for _ in range(10):
        a, b = c0 * np.uint64(PHILOX_M[0]), c2 * np.uint64(PHILOX_M[1])
        c0, c1, c2, c3 = (b >> np.uint64(32)) ^ c1 ^ np.uint64(k0), b & mask, (a >> np.uint64(32)) ^ c3 ^ np.uint64(k1), a & mask
        k0, k1 = (k0 + PHILOX_W[0]) & 0xFFFFFFFF, (k1 + PHILOX_W[1]) & 0xFFFFFFFF
    return np.stack([c0, c1, c2, c3], axis=-1)


def uniforms(seed, layer, kind, slots, heads, dim, step):
    p = padded(dim)
    c0 = np.arange(heads * p // 4, dtype=np.uint64)[None, :]
    w = philox_words(seed, c0, np.uint64(2 * layer + kind), np.asarray(slots, np.uint64)[:, None], np.uint64(step))
    return (w.reshape(len(slots), heads, p)[..., :dim] >> np.uint64(9)).astype(np.float32) * np.float32(2.0 ** -23)


def rotate(x, table, interleaved):
    """fp32 rows [tokens][heads][dim] by table rows [tokens][2 * pairs]; every operation rounded to fp32."""
    x = x.astype(np.float32).copy()
    n = table.shape[1] // 2
    c, s = table[:, None, :n].astype(np.float32), table[:, None, n:].astype(np.float32)
    i, j = (slice(0, 2 * n, 2), slice(1, 2 * n, 2)) if interleaved else (slice(0, n), slice(n, 2 * n))
    a, b = x[..., i].copy(), x[..., j].copy()
    x[..., i], x[..., j] = a * c - b * s, b * c + a * s
    return x


def quantise(x, levels, q, rho):
    """Symbols and norms of fp32 rows [..., dim]."""
    x = x.astype(np.float32)
    with np.errstate(all="ignore"):
        a = np.abs(x)
        a64 = a.astype(np.float64)
        n64 = a64.max(-1) if q == 0 else a64.sum(-1) if q == 1 else np.sqrt(np.square(a64).sum(-1))
        n = n64.astype(np.float32)
        bad = ~np.isfinite(n) | ~np.isfinite(x).all(-1)
        n = np.where(bad | (n < np.float32(2.0 ** -126)), np.float32(0), n)
        inv = np.where(n > 0, np.float32(1) / n, np.float32(0))
        u = np.minimum(np.where(n[..., None] > 0, a * inv[..., None], np.float32(0)), np.float32(1))
        lv = np.asarray(levels, np.float32)
        at = np.minimum(np.searchsorted(lv, u, side="right") - 1, len(lv) - 2)
        up = rho * (lv[at + 1] - lv[at]) < u - lv[at]
        sym = np.where(n[..., None] > 0, 2 * (at + up) + (x < 0), 0)
    return sym.astype(np.uint32), n


def attend(q, k, v, scale, q_error, weight_error):
    """One query [dim] in 64 bits against keys and values [tokens][dim]: out, lse, and bounds of what 32-bit arithmetic, a query of
    relative error q_error and weights of relative error weight_error can be off by (before out is rounded to its type)."""
    if k.shape[0] == 0:
        return np.zeros(v.shape[1]), -np.inf, np.zeros(v.shape[1]), 0.0
    s = scale * (k @ q)
    top = s.max()
    p = np.exp(s - top)
    total = p.sum()
    out = (p @ v) / total
    # a score: q's error on every term, fp32 sums of up to 256 products in steps of 16 (each truncated at 2^-23 of the sum so
    # far), three fp32 factors; its base-2 exponent is one fp32 product and difference of numbers up to |s| and |top|
    size = scale * (np.abs(k) @ np.abs(q))
    off = size * (q_error + 18 * 2.0 ** -23) + (np.abs(s) + abs(top)) * 2.0 ** -22
    # a weight: exp2 and log2 to 2^-21 each, its rounding; sums over tokens in fp32, pairwise over lanes, warps and CTAs
    rel = 2 * off.max() + 2.0 ** -20 + weight_error + (8 + np.sqrt(len(p))) * 2.0 ** -23
    # weights below 2^-20 of the largest lose bits: 2^-31 of it at most
    size_v = np.abs(v).max(0)
    bound = rel * ((p @ np.abs(v)) / total) + len(p) * 2.0 ** -31 * size_v / max(total, 1.0)
    return out, top + np.log(total), bound, off.max() + 2.0 ** -20 + (8 + np.sqrt(len(p))) * 2.0 ** -23 + 2.0 ** -23 * abs(top + np.log(total))
