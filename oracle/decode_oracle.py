"""CPU oracle for the decode-side operators (page map, cache append, page scores and selection, attention of
one new token over a paged cache).

TEST INFRASTRUCTURE ONLY, like cosa_oracle: the plain float64 statement of what include/cosa_decode.h
says, sharing no code with the library or its binding. bf16 data arrives as uint16 bit patterns.
"""
from __future__ import annotations

import math

import numpy as np

from oracle.cosa_oracle import default_scale, widen

I32_MAX = 2 ** 31 - 1


def page_map(cached, new, free, n_free, table, page, max_new):
    """Returns (table, seq_lens, cu_new, slots, n_taken); requests are served in order."""
    table = np.array(table, dtype=np.int64)
    n, width = table.shape
    cap = width * page
    n_free = min(max(int(n_free), 0), len(free))
    seq, cu, slots = [], [0], np.full(max_new, -1, np.int64)
    need_so_far, taken, row = 0, 0, 0
    for r in range(n):
        c, w = min(max(int(cached[r]), 0), cap), max(int(new[r]), 0)
        first_row, row = row, min(row + w, I32_MAX)
        fits = c + w <= cap and first_row + w <= max_new
        first_page, end_page = -(-c // page), -(-(c + w) // page)
        need = end_page - first_page if fits else 0
        base, need_so_far = need_so_far, need_so_far + need
        ok = fits and (need == 0 or need_so_far <= n_free)
        if ok:
            for i in range(need):
                table[r, first_page + i] = free[base + i]
            taken = base + need if need else taken
            for i in range(w):
                pg = table[r, (c + i) // page]
                slots[first_row + i] = pg * page + (c + i) % page if pg >= 0 else -1
        seq.append(c + w if ok else c)
        cu.append(row)
    return table, np.array(seq), np.array(cu), slots, taken


def ordered(bits):
    """bf16 bit patterns as integers in the order of their values (NaN beyond the infinities)."""
    x = np.asarray(bits, dtype=np.uint16).view(np.int16).astype(np.int32)
    return np.where(x < 0, x ^ 0x7FFF, x)


def from_ordered(x):
    return np.where(x < 0, x ^ 0x7FFF, x).astype(np.int16).view(np.uint16)


def kv_append(k_cache, v_cache, bounds, k, v, slots):
    """Writes in place, row after row; caches [pages, Hkv, page, d] bits, bounds [pages, Hkv, 2, d] or None."""
    n_pages, _, page, _ = k_cache.shape
    for t, s in enumerate(slots):
        if not 0 <= s < n_pages * page:
            continue
        p, off = divmod(int(s), page)
        k_cache[p, :, off], v_cache[p, :, off] = k[t], v[t]
        if bounds is not None:
            x = ordered(k[t])
            lo = x if off == 0 else np.minimum(ordered(bounds[p, :, 0]), x)
            hi = x if off == 0 else np.maximum(ordered(bounds[p, :, 1]), x)
            bounds[p, :, 0], bounds[p, :, 1] = from_ordered(lo), from_ordered(hi)


def page_score(q, bounds, table, lens, page, sm_scale=0.0):
    """(score, magnitude) [B, Hq, max_pages] float64, NaN where nothing is written; magnitude: the sum of the
    terms' absolute values, for tolerances."""
    B, Hq, d = q.shape
    scale, g = default_scale(d, sm_scale), Hq // bounds.shape[1]
    out = np.full((B, Hq, table.shape[1]), np.nan)
    mag = out.copy()
    qq, bb = widen(q), widen(bounds)
    for n in range(B):
        for j in range(-(-int(lens[n]) // page)):
            for h in range(Hq):
                lo, hi = bb[table[n, j], h // g]
                terms = np.maximum(qq[n, h] * lo, qq[n, h] * hi)
                out[n, h, j], mag[n, h, j] = scale * terms.sum(), scale * np.abs(terms).sum()
    return out, mag


def kept_pages(p, fraction, min_pages, max_pages, sink, recent):
    micro = math.floor(float(np.float32(fraction)) * 1e6 + 0.5)
    frac = (micro * p + 999999) // 1000000
    return min(p, max(sink + recent, min(max_pages, max(min_pages, frac))))


def page_select(score, lens, page, n_kv_heads, fraction, min_pages, max_pages, sink, recent):
    """(pages [B, Hkv, max_pages], count) from float32 scores; differences in float32 as specified."""
    B, Hq, _ = score.shape
    g = Hq // n_kv_heads
    pages = np.full((B, n_kv_heads, max_pages), -1, np.int64)
    count = np.zeros((B, n_kv_heads), np.int64)
    for n in range(B):
        p = -(-int(lens[n]) // page)
        K = kept_pages(p, fraction, min_pages, max_pages, sink, recent)
        for h in range(n_kv_heads):
            count[n, h] = K
            if p == 0:
                continue
            rows = np.asarray(score[n, h * g:(h + 1) * g, :p], dtype=np.float32)
            with np.errstate(invalid="ignore"):
                top = np.fmax.reduce(rows, axis=1, initial=-np.inf)
                s = (rows - top[:, None].astype(np.float32)).max(0)
            def rank(j):
                forced = j < sink or j >= p - recent
                return (not forced, not np.isnan(s[j]), 0.0 if np.isnan(s[j]) else -float(s[j]), j)
            pages[n, h, :K] = sorted(sorted(range(p), key=rank)[:K])
    return pages, count


def decode_attention(q, k_cache, v_cache, table, lens, pages=None, count=None, sm_scale=0.0):
    """Returns float64 o [B, Hq, d], lse [B, Hq], weight (sum of p |v| per element) and logit magnitude
    (largest scale * sum |q k| per row), the last two for tolerances."""
    B, Hq, d = q.shape
    n_pages, Hkv, page, _ = k_cache.shape
    scale, g = default_scale(d, sm_scale), Hq // Hkv
    o, wt = np.zeros((B, Hq, d)), np.zeros((B, Hq, d))
    lse, mag = np.full((B, Hq), -np.inf), np.zeros((B, Hq))
    qq = widen(q)
    for n in range(B):
        cap = table.shape[1] * page
        length = min(max(int(lens[n]), 0), cap)
        for h in range(Hkv):
            if pages is None:
                logical = list(range(-(-length // page)))
            else:
                c = min(max(int(count[n, h]), 0), pages.shape[2])
                logical = [int(j) for j in pages[n, h, :c] if 0 <= j < table.shape[1] and j * page < length]
            if not logical:
                continue
            at = [int(table[n, j]) if 0 <= table[n, j] < n_pages else 0 for j in logical]
            valid = np.concatenate([np.arange(j * page, (j + 1) * page) < length for j in logical])
            k = widen(k_cache[at, h].reshape(-1, d)[valid])
            v = widen(v_cache[at, h].reshape(-1, d)[valid])
            for hh in range(h * g, (h + 1) * g):
                s = scale * (k @ qq[n, hh])
                m = s.max()
                p = np.exp(s - m)
                o[n, hh] = (p @ v) / p.sum()
                wt[n, hh] = (p @ np.abs(v)) / p.sum()
                lse[n, hh] = m + math.log(p.sum())
                mag[n, hh] = scale * (np.abs(k) @ np.abs(qq[n, hh])).max()
    return o, lse, wt, mag
