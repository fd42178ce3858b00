"""cosa_decode_sparse with budgets above the table's width."""
import numpy as np
import pytest

from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from paper_2607_25291_amd.inputs import f32_to_bf16_bits
from tests.decode_util import Cache, as_f64, check_attention, normal
from tests.gpu_util import dev, torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fraction", [0.3, 1.0])
@pytest.mark.parametrize("page,width,lens,pages", [
    (64, 32, [1500, 40, 0], 1 << 25),       # 2^31 tokens a list, were it that long
    (16, 100, [1600, 777, 3], 101), (16, 100, [1600, 777, 3], 1 << 20), (32, 10, [300, 1, 320], 1 << 26),
])
def test_budgets_above_the_tables_width(page, width, lens, pages, fraction):
    """The fraction alone then says how many pages are kept. The lists have the width of the budget; where a call on
    such lists is possible at all, it gives the same bits."""
    t = torch()
    print(f"[decode budget] page {page} width {width} budget {pages} fraction {fraction}", flush=True)
    rng = np.random.default_rng(width + page)
    c = Cache(rng, lens, 1, page, width)
    kv = c.upload()
    q = normal(rng, len(lens), 20, 128)
    bounds = dev(f32_to_bf16_bits(np.sort(rng.standard_normal((c.n_pages, 1, 2, 128), dtype=np.float32), axis=2)))
    p = B.DecodeProblem(len(lens), 20, 1, width)
    budget = B.page_budget(pages, fraction=fraction, sink_pages=0, recent_pages=0)
    n = B.cosa_decode_sparse_workspace_bytes(p, budget)
    ws = t.empty(n, dtype=t.uint8, device="cuda")
    o = t.full((len(lens), 20, 128), 0x7FC0, dtype=t.int16, device="cuda")
    lse = t.full((len(lens), 20), float("nan"), device="cuda")
    B.cosa_decode_sparse(p, dev(q), kv, bounds, c.lens_d, budget, ws, n, o, lse)
    t.cuda.synchronize()
    lay = B.cosa_decode_sparse_workspace_layout(p, budget)
    lists = ws[lay.pages:lay.pages + 4 * len(lens) * pages].view(t.int32).view(len(lens), 1, pages)
    count = ws[lay.count:lay.count + 4 * len(lens)].view(t.int32).view(len(lens), 1)
    micro = int(np.floor(float(np.float32(fraction)) * 1e6 + 0.5))
    held = [-(-x // page) for x in lens]
    assert count.flatten().tolist() == [-(-micro * h // 1000000) for h in held]
    assert (lists[:, :, width:] == -1).all()
    few = lists[:, :, :width].cpu().numpy()
    ref = D.decode_attention(q, c.k, c.v, c.table, lens, few, count.cpu().numpy())
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, max(lens))
    if pages * page < 2 ** 31:
        o2, lse2 = t.zeros_like(o), t.zeros_like(lse)
        nd = B.cosa_decode_workspace_bytes(p)
        wd = t.empty(nd, dtype=t.uint8, device="cuda")
        B.cosa_decode_attention_listed(p, dev(q), kv, c.lens_d, lists, count, pages, wd, nd, o2, lse2)
        t.cuda.synchronize()
        assert t.equal(o, o2) and t.equal(lse, lse2)
