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
