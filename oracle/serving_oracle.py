"""CPU oracle for the serving operators (attention of chunks of new tokens, and the cache's pages).

TEST INFRASTRUCTURE ONLY, like cosa_oracle: the plain float64 statement of what include/cosa_serving.h says,
sharing no code with the library or its binding. bf16 data arrives as uint16 bit patterns.
"""
from __future__ import annotations

import numpy as np

from oracle.cosa_oracle import default_scale, widen


def chunk_attention(q, k_cache, v_cache, table, lens, cu, sm_scale=0.0):
    """Returns float64 o [rows, Hq, d] (NaN where nothing is written), lse, weight (sum of p |v| per element) and logit
    magnitude (largest scale * sum |q k| per row), the last two for tolerances."""
    rows, Hq, d = q.shape
    n_pages, Hkv, page, _ = k_cache.shape
    scale, g = default_scale(d, sm_scale), Hq // Hkv
    o, wt = np.full((rows, Hq, d), np.nan), np.zeros((rows, Hq, d))
    lse, mag = np.full((rows, Hq), np.nan), np.zeros((rows, Hq))
    cap = table.shape[1] * page
    for n in range(len(lens)):
        a = min(max(int(cu[n]), 0), rows)
        b = min(max(int(cu[n + 1]), a), rows)
        length, w = min(max(int(lens[n]), 0), cap), b - a
        o[a:b], lse[a:b] = 0.0, -np.inf
        if w == 0 or length == 0:
            continue
        at = np.arange(length)
        phys = np.array([int(p) if 0 <= int(p) < n_pages else 0 for p in table[n, :-(-length // page)]])
        pos = length - w + np.arange(w)
        for h in range(Hkv):
            k = widen(k_cache[phys[at // page], h, at % page])
            v = widen(v_cache[phys[at // page], h, at % page])
            for hh in range(h * g, (h + 1) * g):
                qq = widen(q[a:b, hh])
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (qq @ k.T)
                    big = scale * (np.abs(qq) @ np.abs(k).T)
                for i in np.nonzero(pos >= 0)[0]:
                    seen = slice(0, pos[i] + 1)
                    with np.errstate(invalid="ignore", over="ignore"):
                        m = s[i, seen].max()
                        if m == -np.inf:
                            continue
                        p = np.exp(s[i, seen] - m)
                        total = p.sum()
                        o[a + i, hh] = (p @ v[seen]) / total
                        wt[a + i, hh] = (p @ np.abs(v[seen])) / total
                        lse[a + i, hh] = m + np.log(total)
                        mag[a + i, hh] = big[i, seen].max()
    return o, lse, wt, mag


def held(table, lens, page, n_pages):
    """[(row, entry, page)] of the pages that rows hold; entries outside the cache are no pages."""
    cap = table.shape[1] * page
    out = []
    for r in range(table.shape[0]):
        for j in range(-(-min(max(int(lens[r]), 0), cap) // page)):
            if 0 <= int(table[r, j]) < n_pages:
                out.append((r, j, int(table[r, j])))
    return out


def page_fork(parent, table, lens, page, copy_all, free, n_free, new_table):
    """Returns (new_table, new_lens, src, dst, rows): the lists as far as they are written."""
    new_table = np.array(new_table, dtype=np.int64)
    cap = table.shape[1] * page
    n_free = min(max(int(n_free), 0), len(free))
    has_child, lists, new_lens, needed = set(), [], [], 0
    for c, p in enumerate(parent):
        if not 0 <= p < len(lens):
            new_lens.append(0)
            continue
        length = min(max(int(lens[p]), 0), cap)
        pages, part = -(-length // page), length % page
        fresh = None
        if part and (copy_all or p in has_child):
            needed += 1
            if needed > n_free:
                new_lens.append(0)
                continue
            fresh = int(free[needed - 1])
            lists.append((int(table[p, pages - 1]), fresh, part))
        has_child.add(p)
        new_table[c, :pages] = table[p, :pages]
        if fresh is not None:
            new_table[c, pages - 1] = fresh
        new_lens.append(length)
    src, dst, rows = (np.array([x[i] for x in lists], dtype=np.int64) for i in range(3))
    return new_table, np.array(new_lens, dtype=np.int64), src, dst, rows


def page_copy(k_cache, v_cache, bounds, src, dst, rows, n):
    """In place; caches [pages, Hkv, page, d], bounds [pages, Hkv, 2, d] or None, rows or None."""
    n_pages, _, page, _ = k_cache.shape
    for i in range(min(max(int(n), 0), len(src))):
        s, d = int(src[i]), int(dst[i])
        if not (0 <= s < n_pages and 0 <= d < n_pages):
            continue
        keep = page if rows is None else min(max(int(rows[i]), 0), page)
        k_cache[d, :, :keep], v_cache[d, :, :keep] = k_cache[s, :, :keep], v_cache[s, :, :keep]
        if bounds is not None:
            bounds[d] = bounds[s]


def page_release(old_table, old_lens, new_table, new_lens, page, n_pages, free, n_free, n_taken):
    """The free list afterwards."""
    n_free = min(max(int(n_free), 0), len(free))
    left = [int(p) for p in free[min(max(int(n_taken), 0), n_free):n_free]]
    old = {p for _, _, p in held(old_table, old_lens, page, n_pages)}
    new = {p for _, _, p in held(new_table, new_lens, page, n_pages)}
    return left + sorted(old - new - set(left))


def page_compact(table, lens, page, n_pages, max_moves):
    """Returns (new table, moves [(src, dst)], free list)."""
    table = np.array(table, dtype=np.int64)
    entries = held(table, lens, page, n_pages)
    used = sorted({p for _, _, p in entries})
    unused = sorted(set(range(n_pages)) - set(used))
    moves = []
    for s, d in zip(reversed(used), unused):
        if d > s or len(moves) == max_moves:
            break
        moves.append((s, d))
    to = dict(moves)
    for r, j, p in entries:
        table[r, j] = to.get(p, p)
    now = {to.get(p, p) for p in used}
    return table, moves, [p for p in range(n_pages) if p not in now]
