"""Attention of one new token where a group's heads take several units and the join's last workgroup of a unit has
more room than the unit has heads: over all pages, over lists and over selected pages, against the float64
oracle."""
import sys

import numpy as np
import pytest

from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, as_f64, check_attention, normal, run_decode
from tests.gpu_util import dev, torch

pytestmark = pytest.mark.gpu

# name: (sequences, longest, query heads, KV heads, page, table width in pages): units, heads a join workgroup, rows
CASES = {
    "g20_17": (17, 1500, 20, 1, 16, 94),       # 34 units of 16 rows, 3 heads
    "g20_34": (34, 1500, 20, 1, 16, 94),       # 68 units of 16 rows, 6 heads
    "g20_5x4": (5, 2000, 80, 4, 64, 32),       # 40 units of 16 rows, 3 heads
    "g17_21x2": (21, 1400, 34, 2, 128, 11),    # 84 units of 16 rows, 6 heads
    "g40_18": (18, 3000, 40, 1, 64, 64),       # 36 units of 32 rows, 5 heads
    "g33_9": (9, 5000, 33, 1, 64, 120),        # 18 units of 32 rows, 3 heads
    "g70_12": (12, 2000, 70, 1, 32, 180),      # 36 units of 32 rows, 5 heads
}


def inputs(name):
    batch, longest, hq, hkv, page, width = CASES[name]
    print(f"[decode join] {name}", flush=True)
    sys.stdout.flush()
    rng = np.random.default_rng(len(name) + batch)
    lens = [longest] + [int(x) for x in rng.integers(0, longest + 1, batch - 1)]
    c = Cache(rng, lens, hkv, page, width)
    return rng, lens, c, normal(rng, batch, hq, 128), B.DecodeProblem(batch, hq, hkv, width)


def check(o, lse, ref, longest):
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, longest)


@pytest.mark.parametrize("name", list(CASES))
def test_all_pages(name):
    _, lens, c, q, p = inputs(name)
    o, lse = run_decode(p, c, dev(q))
    check(o, lse, D.decode_attention(q, c.k, c.v, c.table, lens), max(lens))


@pytest.mark.parametrize("name", list(CASES))
def test_listed_pages(name):
    rng, lens, c, q, p = inputs(name)
    pages = np.full((p.batch, p.n_kv_heads, c.width), -1, np.int32)
    count = np.zeros((p.batch, p.n_kv_heads), np.int32)
    for n, length in enumerate(lens):
        have = -(-length // c.page)
        for h in range(p.n_kv_heads):
            k = int(rng.integers(0, have + 1))
            pages[n, h, :k] = rng.permutation(have)[:k]
            count[n, h] = k
    o, lse = run_decode(p, c, dev(q), (pages, count))
    check(o, lse, D.decode_attention(q, c.k, c.v, c.table, lens, pages, count), max(lens))


@pytest.mark.parametrize("name", list(CASES))
def test_selected_pages(name):
    t = torch()
    rng, lens, c, q, p = inputs(name)
    kv = c.upload()
    bounds = np.sort(rng.standard_normal((c.n_pages, p.n_kv_heads, 2, 128), dtype=np.float32), axis=2)
    from paper_2607_25291_amd.inputs import f32_to_bf16_bits
    budget = B.page_budget(c.width - 1, sink_pages=1, recent_pages=1)
    n = B.cosa_decode_sparse_workspace_bytes(p, budget)
    ws = t.full((n,), 0xFF, dtype=t.uint8, device="cuda")
    o = t.full((p.batch, p.n_q_heads, 128), 0x7FC0, dtype=t.int16, device="cuda")
    lse = t.full((p.batch, p.n_q_heads), float("nan"), device="cuda")
    B.cosa_decode_sparse(p, dev(q), kv, dev(f32_to_bf16_bits(bounds)), c.lens_d, budget, ws, n, o, lse)
    t.cuda.synchronize()
    lay = B.cosa_decode_sparse_workspace_layout(p, budget)
    rows = p.batch * p.n_kv_heads
    pages = ws[lay.pages:lay.pages + 4 * rows * budget.max_pages].view(t.int32).view(p.batch, p.n_kv_heads, -1).cpu().numpy()
    count = ws[lay.count:lay.count + 4 * rows].view(t.int32).view(p.batch, p.n_kv_heads).cpu().numpy()
    assert count.max() == min(-(-max(lens) // c.page), budget.max_pages)
    check(o, lse, D.decode_attention(q, c.k, c.v, c.table, lens, pages, count), max(lens))
