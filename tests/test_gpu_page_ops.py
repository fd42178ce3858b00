"""Page maps, cache append with key bounds, page scores and page selection against the oracle."""
import sys

import numpy as np
import pytest

from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, normal
from tests.gpu_util import dev, host_bits, torch

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


# ---- page map

def page_map(cached, new, free, n_free, table, page, max_new):
    t = torch()
    n, width = table.shape
    i32 = lambda x: dev(np.asarray(x, np.int32))
    table_d, free_d = i32(table), i32(free)
    seq, cu = t.full((n,), -7, dtype=t.int32, device="cuda"), t.full((n + 1,), -7, dtype=t.int32, device="cuda")
    slots = t.full((max_new + 3,), -7, dtype=t.int64, device="cuda")
    taken = t.full((1,), -7, dtype=t.int32, device="cuda")
    B.cosa_page_map(n, page, width, i32(cached), i32(new), free_d, len(free), i32([n_free]), table_d, seq, cu, slots,
                    max_new, taken)
    t.cuda.synchronize()
    assert (slots[max_new:] == -7).all()
    return tuple(x.cpu().numpy() for x in (table_d, seq, cu, slots[:max_new])) + (int(taken.item()),)


def check_map(*args):
    got, want = page_map(*args), D.page_map(*args)
    for name, a, b in zip(("table", "seq_lens", "cu_new", "slots", "n_taken"), got, want):
        assert np.array_equal(a, b), name


@pytest.mark.parametrize("batch,page,width,new,pool", [
    (1, 16, 1, 1, 4), (1, 64, 40, 2000, 40), (3, 16, 8, 1, 8), (64, 64, 30, 1, 70), (257, 16, 20, 300, 9000),
    (257, 16, 20, 300, 2000), (1000, 128, 6, 700, 6000), (8192, 16, 3, 40, 20000), (5, 1 << 20, 3, 70000, 9),
])
def test_page_map(batch, page, width, new, pool):
    say(f"[page map] batch {batch} page {page} width {width} new {new} pool {pool}")
    rng = np.random.default_rng(batch + new)
    cap = width * page
    cached = rng.integers(0, cap + 1, batch) * (rng.random(batch) < 0.7)
    add = np.minimum(rng.integers(0, new + 1, batch), cap - cached + (rng.random(batch) < 0.05))
    free = rng.permutation(2 * pool)[:pool]
    table = np.where(np.arange(width)[None] * page < cached[:, None], rng.integers(0, 2 ** 20, (batch, width)), -1)
    total = int(add.sum())
    check_map(cached, add, free, pool, table, page, total + 5)
    check_map(cached, add, free, pool // 3, table, page, max(total - 7, 0))


def test_page_map_odd_values():
    """Negative and huge lengths, a pool count outside its list, nothing to add, no rows and no pages."""
    table = np.array([[3, -1], [-5, 8], [2, 9], [1, 1], [4, 6]])
    args = ([-3, 5, 2 ** 31 - 1, 20, 0], [4, 9, 1, -2, 2 ** 31 - 1], [10, 11, 12])
    for n_free in (-1, 0, 1, 3, 100):
        check_map(*args, n_free, table, 16, 40)
    check_map([0, 40, 33], [0, 0, 0], [], 5, np.full((3, 3), 2), 16, 4)
    check_map([0], [3], [1], 1, np.zeros((1, 0)), 16, 4)
    check_map([5], [3], [1], 1, np.zeros((1, 2)), 16, 0)
    # rows that pass 2^31 - 1: the prefix sums stay there
    check_map([0] * 3, [2 ** 31 - 1, 2 ** 31 - 1, 1], [1, 2], 2, np.zeros((3, 2)), 16, 8)


# ---- cache append

def append(heads, page, kc, vc, bounds, k, v, slots, **kw):
    t = torch()
    d = [dev(x) for x in (kc, vc)] + [None if bounds is None else dev(bounds)]
    B.cosa_kv_append(heads, 128, page, kc.shape[0], d[0], d[1], d[2], len(slots), k, v,
                     dev(np.asarray(slots, np.int64)), **kw)
    t.cuda.synchronize()
    return [None if x is None else host_bits(x) for x in d]


def check_append(heads, page, kc, vc, bounds, k, v, slots):
    got = append(heads, page, kc, vc, bounds, dev(k), dev(v), slots)
    kc, vc = kc.copy(), vc.copy()
    want_b = None if bounds is None else bounds.copy()
    D.kv_append(kc, vc, want_b, k, v, slots)
    assert np.array_equal(got[0], kc) and np.array_equal(got[1], vc)
    if bounds is not None:
        assert np.array_equal(got[2], want_b)


@pytest.mark.parametrize("with_bounds", [True, False])
@pytest.mark.parametrize("heads,page,lens,new", [
    (1, 16, [1], [1]), (2, 16, [16, 17, 33], [1, 1, 1]), (8, 64, [64, 65, 100, 1, 128], [64, 1, 36, 1, 65]),
    (5, 32, [700, 3, 90], [650, 0, 90]), (8, 256, [1100, 255], [1001, 254]), (2, 128, [5000] * 3, [4900, 77, 1]),
    (1, 512, [513, 1500, 30], [513, 700, 1]), (3, 2048, [4100, 2040, 2050], [3000, 1, 5]), (1, 16, [9000] * 4, [8999] * 4),
])
def test_append(heads, page, lens, new, with_bounds):
    say(f"[append] heads {heads} page {page} lens {lens} new {new}")
    rng = np.random.default_rng(sum(lens))
    c = Cache(rng, lens, heads, page, spare=2)
    k, v = normal(rng, sum(new), heads, 128), normal(rng, sum(new), heads, 128)
    k[:, :, 3] = 0x8000   # -0 beside +0
    k[::2, :, 3] = 0
    slots = np.concatenate([[c.table[n, (s - w + i) // page] * page + (s - w + i) % page for i in range(w)]
                            for n, (s, w) in enumerate(zip(lens, new))] + [[]]).astype(np.int64)
    bounds = rng.integers(0, 2 ** 16, (c.n_pages, heads, 2, 128), dtype=np.uint16) if with_bounds else None
    check_append(heads, page, c.k, c.v, bounds, k, v, slots)


def test_append_skips_and_scattered_slots():
    """Padding (-1) and foreign slots among real ones leave everything else as it was; without bounds any
    order of slots is right; NaN and infinite keys."""
    rng = np.random.default_rng(3)
    kc, vc = normal(rng, 6, 3, 16, 128), normal(rng, 6, 3, 16, 128)
    b = normal(rng, 6, 3, 2, 128)
    k, v = normal(rng, 200, 3, 128), normal(rng, 200, 3, 128)
    k[0, 0, :3] = [0x7FC0, 0xFFC0, 0x7F80]
    k[1, 1, :2] = [0xFF80, 0x7F80]
    slots = np.full(200, -1, np.int64)
    slots[:20] = np.arange(32, 52)                  # page 2 from its start into page 3
    slots[30:36] = np.arange(85, 91)                # page 5, behind tokens that were there
    slots[60], slots[199] = 96, 2 ** 40             # just outside, far outside
    slots[100] = -2 ** 62
    check_append(3, 16, kc, vc, b, k, v, slots)
    slots = rng.permutation(96)
    check_append(3, 16, kc, vc, None, k[:96], v[:96], slots)


def test_append_strided_rows():
    rng = np.random.default_rng(4)
    kc, vc, b = normal(rng, 4, 2, 16, 128), normal(rng, 4, 2, 16, 128), normal(rng, 4, 2, 2, 128)
    wide = normal(rng, 37, 12, 128)
    slots = np.arange(20, 57)
    d = dev(wide)
    got = append(2, 16, kc, vc, b, d[:, 8:10], d[:, 10:12], slots)
    D.kv_append(kc, vc, b, np.ascontiguousarray(wide[:, 8:10]), np.ascontiguousarray(wide[:, 10:12]), slots)
    for x, y in zip(got, (kc, vc, b)):
        assert np.array_equal(x, y)


# ---- page scores

@pytest.mark.parametrize("lens,hq,hkv,page,width", [
    ([1], 1, 1, 16, None), ([0, 16, 17, 255, 256, 257], 4, 2, 16, 40), ([4000, 700], 28, 4, 64, None),
    ([1025, 33], 17, 1, 16, 101), ([9000], 80, 2, 32, 300), ([600] * 9, 5, 5, 128, None),
])
def test_page_score(lens, hq, hkv, page, width):
    say(f"[page score] lens {lens} hq {hq} hkv {hkv} page {page}")
    t = torch()
    rng = np.random.default_rng(hq + page)
    c = Cache(rng, lens, hkv, page, width)
    kv = c.upload()
    bounds = np.sort(rng.standard_normal((c.n_pages, hkv, 2, 128), dtype=np.float32), axis=2)
    from paper_2607_25291_amd.inputs import f32_to_bf16_bits
    bounds = f32_to_bf16_bits(bounds + 0.3 * rng.standard_normal((c.n_pages, hkv, 1, 128), dtype=np.float32))
    wide = normal(rng, len(lens), hq + 3, 128)
    wide[0, 1, :4] = [0, 0x8000, 0, 0x8000]
    q = np.ascontiguousarray(wide[:, 1:1 + hq])
    score = t.full((len(lens), hq, c.width), float("nan"), device="cuda")
    B.cosa_page_score(B.DecodeProblem(len(lens), hq, hkv, c.width), dev(wide)[:, 1:1 + hq], kv, dev(bounds),
                      c.lens_d, score)
    got = score.cpu().numpy().astype(np.float64)
    want, mag = D.page_score(q, bounds, c.table, lens, page)
    assert (np.isnan(got) == np.isnan(want)).all()  # nothing written behind a sequence's pages
    live = ~np.isnan(want)
    # fp32 sums of 256 exact products (128 of them zero): 256 * 2^-24 of the magnitudes, and the scale's rounding
    assert (np.abs(got - want)[live] <= (2.0 ** -16 + 2.0 ** -22) * mag[live]).all()


# ---- selection

def select(score, lens, page, hkv, budget):
    t = torch()
    n, hq, width = score.shape
    pages = t.full((n, hkv, budget.max_pages), -7, dtype=t.int32, device="cuda")
    count = t.full((n, hkv), -7, dtype=t.int32, device="cuda")
    B.cosa_page_select(B.DecodeProblem(n, hq, hkv, width), page, dev(np.asarray(lens, np.int32)), dev(score), budget,
                       pages, count)
    t.cuda.synchronize()
    return pages.cpu().numpy(), count.cpu().numpy()


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("lens,hq,hkv,page,width,budget", [
    ([1], 1, 1, 16, 1, dict(max_pages=2, sink_pages=0, recent_pages=0)),
    ([0, 1, 16, 17, 200, 256], 4, 2, 16, 16, dict(max_pages=6)),
    ([640, 4000, 64], 8, 8, 64, 63, dict(max_pages=20, min_pages=3, fraction=0.2)),
    ([131072, 70000, 3], 28, 4, 32, 4096, dict(max_pages=300, sink_pages=2, recent_pages=5)),
    ([131072], 17, 1, 16, 8192, dict(max_pages=1000, min_pages=1000, sink_pages=0, recent_pages=0)),
    ([524288, 500001], 2, 1, 16, 32768, dict(max_pages=700, fraction=0.01, sink_pages=1, recent_pages=3)),
    ([4000, 100], 16, 2, 16, 250, dict(max_pages=40, sink_pages=1, recent_pages=2)),
    ([5000] * 30, 5, 5, 16, 400, dict(max_pages=313, sink_pages=0, recent_pages=1)),
])
def test_page_select(lens, hq, hkv, page, width, budget, ties):
    say(f"[page select] lens {lens[:4]} hq {hq} hkv {hkv} page {page} budget {budget} ties {ties}")
    rng = np.random.default_rng(width + ties)
    score = rng.standard_normal((len(lens), hq, width)).astype(np.float32) * 3 + 5
    if ties:
        score = np.round(score * 2) / 2
    for n, length in enumerate(lens):
        score[n, :, -(-length // page):] = np.nan  # not part of the row
    b = B.page_budget(**budget)
    got = select(score, lens, page, hkv, b)
    want = D.page_select(score, lens, page, hkv, b.fraction, b.min_pages, b.max_pages, b.sink_pages, b.recent_pages)
    assert np.array_equal(got[1], want[1])
    assert np.array_equal(got[0], want[0])


def test_page_select_odd_scores():
    """All equal, infinities, NaN, and zeros of either sign."""
    rng = np.random.default_rng(0)
    score = rng.standard_normal((6, 3, 50)).astype(np.float32)
    score[0] = 2.5
    score[1, 0, 7], score[1, 1, 9] = np.inf, -np.inf
    score[2, 2, 30:33] = np.nan
    score[3] = -np.inf
    score[4, :, ::2], score[4, :, 1::2] = 0.0, -0.0
    score[5, 1] = np.nan
    lens = [50 * 16] * 6
    for keep in (1, 5, 49, 50, 60):
        b = B.page_budget(keep, sink_pages=0, recent_pages=0)
        got = select(score, lens, 16, 1, b)
        want = D.page_select(score, lens, 16, 1, 1.0, 1, keep, 0, 0)
        assert np.array_equal(got[1], want[1])
        assert np.array_equal(got[0], want[0]), keep
