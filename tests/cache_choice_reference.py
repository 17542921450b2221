"""Bounds of a page's keys and the choice of pages by them, in numpy, from their definition (tests only)."""
import numpy as np

import cache_reference as R

F = np.float32
LEAST = F(2.0 ** -100)


def bounds(pages, heads, dim, page, bits, levels):
    """pages uint32 [n][words] -> upper, lower int [n][heads][padded], scales fp32 [n][heads]."""
    sym, _, norms, _ = R.head_sections(pages, heads, dim, page, bits)
    with np.errstate(all="ignore"):
        v = (np.asarray(levels, F)[sym >> 1] * np.where(sym & 1, F(-1), F(1))).astype(F) * norms[..., None]       # fp32 products
        n = norms.max(-1)
        kept = (n >= LEAST) & np.isfinite(norms).all(-1)
        inv = np.where(kept, F(127) * (F(1) / np.where(kept, n, F(1))), F(0)).astype(F)[..., None]
        up = np.clip(np.ceil(np.nan_to_num(v.max(2)) * inv), -127, 127)
        low = np.clip(np.floor(np.nan_to_num(v.min(2)) * inv), -127, 127)
    up, low = (np.where(kept[..., None], x, 0).astype(np.int64) for x in (up, low))
    return up, low, np.where(kept, n * (F(1) / F(127)), F(0)).astype(F)


def unpacked(words, heads, padded):
    """Rows of a bounds buffer, uint32 [n][words] -> upper, lower, scales as above."""
    b = words[:, : heads * padded // 2].copy().view(np.int8).reshape(len(words), heads, 2, padded).astype(np.int64)
    return b[:, :, 0], b[:, :, 1], words[:, heads * padded // 2: heads * padded // 2 + heads].copy().view(F)


def whole(q):
    """fp32 queries [..., dim] -> whole numbers and scales."""
    q = q.astype(F)
    with np.errstate(all="ignore"):
        top = np.where(np.isnan(q).any(-1), F(np.inf), np.abs(np.nan_to_num(q, nan=0.0, posinf=np.inf, neginf=-np.inf)).max(-1)).astype(F)
        kept = (top >= LEAST) & np.isfinite(top)
        inv = np.where(kept, F(127) * (F(1) / np.where(kept, top, F(1))), F(0)).astype(F)[..., None]
        i = np.where(kept[..., None], np.rint((np.nan_to_num(q) * inv).astype(F)), 0).astype(np.int64)
    return i, np.where(kept, top * (F(1) / F(127)), F(0)).astype(F)


def scores(i, per, up, low, scale):
    """One head: queries [group][dim], [group]; pages [n][dim] twice, [n] -> [n]."""
    dots = np.maximum(i[:, None] * up[None], i[:, None] * low[None]).sum(-1)
    with np.errstate(all="ignore"):
        return ((dots.astype(F) * per[:, None]).astype(F) * scale[None]).astype(F).max(0)


def choose(score, pages, first, last, keep):
    """score [pages] of one head -> indices kept, in order; ties go to the lowest."""
    if pages <= keep:
        return list(range(pages))
    middle = list(range(first, pages - last))
    best = sorted(middle, key=lambda x: (-score[x], x))[: keep - first - last]
    return list(range(first)) + sorted(best) + list(range(pages - last, pages))
