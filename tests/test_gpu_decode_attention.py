"""Attention of one new token over a paged cache against the float64 oracle: lengths from none to long,
page sizes, head layouts, lists, garbage behind every sequence, strides, streams and graphs."""
import sys

import numpy as np
import pytest

from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, as_f64, check_attention, normal, run_decode
from tests.gpu_util import dev, torch

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


# name: (lengths, Hq, Hkv, page, table width in pages or None). Lengths around the 16-key halves, the 128-token tiles,
# page ends and the split; batches that leave workgroups several units, part of one, or none.
CASES = {
    "one_token": ([1], 1, 1, 16, None),
    "tiny_mix": ([0, 1, 2, 15, 16, 17, 31, 33, 127, 128, 129], 4, 2, 16, None),
    "wide_table": ([5, 0, 300], 8, 2, 16, 4096),
    "one_head_1k": ([1000], 1, 1, 32, None),
    "gqa4": ([1537, 64, 0, 777, 4001], 32, 8, 64, None),
    "gqa7": ([515, 2049, 130], 28, 4, 128, None),
    "gqa16": ([900, 1300], 32, 2, 16, None),
    "gqa17": ([700, 33], 17, 1, 32, None),
    "gqa40": ([1111, 129, 640], 80, 2, 64, None),
    "mha": ([640, 511, 513, 1], 5, 5, 256, None),
    "one_page": ([3000], 8, 1, 4096, None),
    "many_short": ([1 + 7 * i % 90 for i in range(300)], 8, 4, 16, 64),
    "long_one": ([20000], 4, 1, 128, None),
    "gqa20": ([1300, 70, 5000], 40, 2, 32, None),
    "gqa32": ([4100], 32, 1, 128, None),
    "gqa24_wide": ([4100, 900, 33], 48, 2, 64, 400),   # 32 columns: more tiles than workgroups
    "gqa70_wide": ([1500, 300], 70, 1, 32, 1100),
    # more sequences than lanes and than threads, split (tables of more than 1024 tokens)
    "many_mixed": ([1 + 37 * i % 2600 for i in range(90)], 4, 1, 64, None),
    # 32 columns, units unsplit; split with more units than the join gives heads of their own
    "many_short_wide": ([1 + 11 * i % 500 for i in range(260)], 20, 1, 16, 32),
    "many_wide": ([1 + 29 * i % 1300 for i in range(140)], 48, 2, 64, 24),
    "very_many": ([1 + 13 * i % 41 for i in range(1100)], 2, 1, 16, 70),
    "batch_mixed": ([1, 6000, 40, 2500, 0, 129, 9000, 300], 8, 2, 32, None),
}


@pytest.mark.parametrize("name", list(CASES))
def test_all_pages(name):
    lens, hq, hkv, page, width = CASES[name]
    say(f"[decode] {name}: lens {lens[:12]} hq {hq} hkv {hkv} page {page}")
    rng = np.random.default_rng(len(name) + 1000)
    c = Cache(rng, lens, hkv, page, width)
    q = normal(rng, len(lens), hq, 128)
    p = B.DecodeProblem(len(lens), hq, hkv, c.width)
    o, lse = run_decode(p, c, dev(q))
    ref = D.decode_attention(q, c.k, c.v, c.table, lens)
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, max(lens))
    # again, without lse: the same bits
    o2, _ = run_decode(p, c, dev(q), lse=False)
    assert torch().equal(o, o2)


@pytest.mark.parametrize("name", ["tiny_mix", "gqa4", "gqa17", "gqa20", "gqa24_wide", "batch_mixed", "many_short",
                                  "many_mixed", "many_short_wide", "many_wide"])
def test_listed_pages(name):
    lens, hq, hkv, page, width = CASES[name]
    say(f"[decode listed] {name}")
    rng = np.random.default_rng(len(name) + 2000)
    c = Cache(rng, lens, hkv, page, width)
    q = normal(rng, len(lens), hq, 128)
    p = B.DecodeProblem(len(lens), hq, hkv, c.width)
    n_max = max(3, c.width // 2)
    pages = np.full((len(lens), hkv, n_max), -7, np.int32)
    count = np.zeros((len(lens), hkv), np.int32)
    for n, length in enumerate(lens):
        have = -(-length // page)
        for h in range(hkv):
            k = int(rng.integers(0, min(have, n_max) + 1))
            pages[n, h, :k] = rng.permutation(have)[:k]
            count[n, h] = k
    # entries that add nothing: negative, behind the end, outside the table; counts outside the width
    pages[0, 0, :3] = [-1, 2 ** 31 - 1, c.width]
    count[0, 0] = 3
    if hkv > 1:
        count[-1, -1] = -5
    o, lse = run_decode(p, c, dev(q), (pages, count))
    ref = D.decode_attention(q, c.k, c.v, c.table, lens, pages, count)
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, n_max * page)
    count[-1, 0] = n_max + 100  # read as n_max
    pages[-1, 0] = -1
    pages[-1, 0, 0] = 0
    o, lse = run_decode(p, c, dev(q), (pages, count))
    ref = D.decode_attention(q, c.k, c.v, c.table, lens, pages, count)
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, n_max * page)


def test_list_of_all_pages_matches_the_whole_walk():
    rng = np.random.default_rng(5)
    lens = [700, 2000, 0, 17]
    c = Cache(rng, lens, 2, 32)
    q = normal(rng, 4, 8, 128)
    p = B.DecodeProblem(4, 8, 2, c.width)
    pages = np.tile(np.arange(c.width, dtype=np.int32), (4, 2, 1))
    count = np.array([[-(-n // 32)] * 2 for n in lens], np.int32)
    o, lse = run_decode(p, c, dev(q))
    o2, lse2 = run_decode(p, c, dev(q), (pages, count))
    # twice the same values up to the order of fp32 sums, each rounded to bf16 once: one step at most
    a, b = as_f64(o), as_f64(o2)
    assert (np.abs(a - b) <= 2.0 ** -7 * np.maximum(np.abs(a), np.abs(b)) + 2.0 ** -12).all()
    assert torch().equal(torch().isneginf(lse), torch().isneginf(lse2))


def test_walks_of_many_steps():
    """Lists long enough that a wave looks up its pages more than once: three pages, each listed 100000 times, have the
    weights of the three pages listed once, and a sum 100000 times as large."""
    t = torch()
    rng = np.random.default_rng(11)
    c = Cache(rng, [44], 1, 16, spare=1)
    q = normal(rng, 1, 3, 128)
    p = B.DecodeProblem(1, 3, 1, c.width)
    pages = np.tile(np.arange(3, dtype=np.int32), (1, 1, 100000))
    say(f"[decode steps] a list of {pages.size} pages")
    o, lse = run_decode(p, c, dev(q), (pages, np.full((1, 1), pages.size, np.int32)))
    ro, rl, wt, mag = D.decode_attention(q, c.k, c.v, c.table, [44])
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), (ro, rl + np.log(100000.0), wt, mag),
                    pages.size * 16)
    assert t.isfinite(lse).all()


def test_lengths_and_tables_outside_their_range():
    """Negative lengths are 0, lengths above the table's width are the width; foreign table entries are page 0."""
    rng = np.random.default_rng(6)
    lens = [96, 96, 96]
    c = Cache(rng, lens, 2, 32, sinks=False)
    q = normal(rng, 3, 4, 128)
    p = B.DecodeProblem(3, 4, 2, 3)
    c.lens = np.array([-4, 1000, 96], np.int32)
    zero = c.table[2, 1]
    c.table[2, 1] = -9
    # page 0 must hold numbers: it is read in place of the foreign entry
    c.k[0], c.v[0] = normal(rng, 2, 32, 128), normal(rng, 2, 32, 128)
    o, lse = run_decode(p, c, dev(q))
    ref = D.decode_attention(q, c.k, c.v, c.table, [0, 96, 96])
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, 96)
    assert zero != -9


def test_strided_queries_scale_and_large_logits():
    rng = np.random.default_rng(7)
    lens = [333, 1200]
    c = Cache(rng, lens, 2, 64)
    wide = normal(rng, 2, 24, 128, scale=6.0)
    p = B.DecodeProblem(2, 8, 2, c.width, sm_scale=0.25)
    wide_d = dev(wide)
    q = wide_d[:, 8:16]
    assert not q.is_contiguous()
    o, lse = run_decode(p, c, q)
    ref = D.decode_attention(np.ascontiguousarray(wide[:, 8:16]), c.k, c.v, c.table, lens, sm_scale=0.25)
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, 1200)
    with pytest.raises(ValueError):
        run_decode(p, c, wide_d[:, :8, :64])


def test_infinite_and_nan_values_stay_where_they_are():
    """A NaN value reaches the rows that attend to it and no others; a key at minus infinity has no weight."""
    t = torch()
    rng = np.random.default_rng(8)
    lens = [200, 200]
    c = Cache(rng, lens, 2, 16)
    q = normal(rng, 2, 4, 128)
    p = B.DecodeProblem(2, 4, 2, c.width)
    c.v[c.table[0, 3], 1, 5, 17] = 0x7FC0
    o, _ = run_decode(p, c, dev(q))
    got = (o.cpu().numpy().view(np.uint16) & 0x7FFF) > 0x7F80
    want = np.zeros_like(got)
    want[0, 2:4, 17] = True
    assert (got == want).all()
    # keys of -inf in one dimension, where every query is positive: logits of -inf
    c = Cache(rng, lens, 2, 16)
    q[:, :, 9] = 0x3F80
    c.k[c.table[1, 2], 0, 4:9, 9] = 0xFF80
    o, lse = run_decode(p, c, dev(q))
    with np.errstate(invalid="ignore"):
        ro, rl, wt, mag = D.decode_attention(q, c.k, c.v, c.table, lens)
    c.k[c.table[1, 2], 0, 4:9, 9] = 0
    mag = D.decode_attention(q, c.k, c.v, c.table, lens)[3]
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), (ro, rl, wt, mag), 200)
    assert t.isfinite(lse).all()


@pytest.mark.parametrize("width", [8, 200])  # unsplit, and split over workgroups
def test_nan_logits_are_not_hidden(width):
    """A sequence whose only logits are NaN gives NaN, not the zeros of an empty one; a NaN query its own head."""
    rng = np.random.default_rng(12)
    c = Cache(rng, [1, 0, 700 if width > 8 else 100], 2, 16, width)
    q = normal(rng, 3, 4, 128)
    c.k[c.table[0, 0], 0, 0, 7] = 0x7FC0          # heads 0 and 1 of sequence 0
    q[2, 3, 100] = 0xFFC0                         # head 3 of sequence 2
    p = B.DecodeProblem(3, 4, 2, c.width)
    o, lse = run_decode(p, c, dev(q))
    nan = np.isnan(as_f64(o))
    want = np.zeros_like(nan)
    want[0, :2] = want[2, 3] = True
    assert (nan == want).all()
    assert (np.isnan(lse.cpu().numpy()) == want[..., 0]).all()
    assert (as_f64(o)[1] == 0).all() and np.isneginf(lse.cpu().numpy()[1]).all()


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes per tensor, the used pages at its far end."""
    t = torch()
    rng = np.random.default_rng(9)
    lens = [300, 45]
    c = Cache(rng, lens, 2, 64, spare=0)
    far = (2 ** 32 + 2 ** 26) // (2 * 64 * 128 * 2)
    n_pages = far + c.n_pages
    say(f"[decode far] {n_pages} pages of {2 * 64 * 128 * 2} bytes")
    big = [t.zeros((n_pages, 2, 64, 128), dtype=t.int16, device="cuda") for _ in range(2)]
    for x, y in zip(big, (c.k, c.v)):
        x[far:] = dev(y)
    table = np.where(c.table < c.n_pages, c.table + far, c.table).astype(np.int32)
    table_d = dev(table)
    c.lens_d = dev(c.lens)
    q = normal(rng, 2, 8, 128)
    p = B.DecodeProblem(2, 8, 2, c.width)
    kv = B.paged_kv(big[0], big[1], table_d, 64, n_pages)
    o, lse = run_decode(p, c, dev(q), kv=kv)
    ref = D.decode_attention(q, c.k, c.v, c.table, lens)
    check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, 300)


def test_two_streams_and_a_replayed_graph():
    """Calls on two streams with workspaces of their own, and a captured call replayed after its inputs have changed,
    with eager calls in between: each equals the eager result bit for bit."""
    t = torch()
    rng = np.random.default_rng(10)
    lens = [900, 64, 2100]
    c = Cache(rng, lens, 2, 32, width=100)
    kv = c.upload()
    p = B.DecodeProblem(3, 8, 2, 100)
    qs = [dev(normal(rng, 3, 8, 128)) for _ in range(3)]
    want = [run_decode(p, c, q, kv=kv)[0] for q in qs]
    n = B.cosa_decode_workspace_bytes(p)
    s1, s2 = t.cuda.Stream(), t.cuda.Stream()
    ws = [t.empty(n, dtype=t.uint8, device="cuda") for _ in range(2)]
    out = [t.zeros_like(want[0]) for _ in range(2)]
    t.cuda.synchronize()
    for _ in range(4):
        for s, w, o, q in zip((s1, s2), ws, out, qs):
            B.cosa_decode_attention(p, q, kv, c.lens_d, w, n, o, stream=s)
    t.cuda.synchronize()
    assert t.equal(out[0], want[0]) and t.equal(out[1], want[1])

    q, o = qs[0].clone(), t.zeros_like(want[0])
    side = t.cuda.Stream()
    side.wait_stream(t.cuda.current_stream())
    with t.cuda.stream(side):
        B.cosa_decode_attention(p, q, kv, c.lens_d, ws[0], n, o)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        B.cosa_decode_attention(p, q, kv, c.lens_d, ws[0], n, o)
    for turn in range(4):
        q.copy_(qs[turn % 3])
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(o, want[turn % 3])
        assert t.equal(run_decode(p, c, qs[(turn + 1) % 3], kv=kv)[0], want[(turn + 1) % 3])
    # a second graph of the same workspace, the two replayed in turn
    o2 = t.zeros_like(o)
    graph2 = t.cuda.CUDAGraph()
    with t.cuda.graph(graph2):
        B.cosa_decode_attention(p, qs[2], kv, c.lens_d, ws[0], n, o2)
    q.copy_(qs[0])
    for _ in range(3):
        o.zero_()
        o2.zero_()
        graph2.replay()
        graph.replay()
        t.cuda.synchronize()
        assert t.equal(o, want[0]) and t.equal(o2, want[2])
    # other lengths, same graph
    c.lens_d.copy_(dev(np.array([0, 64, 1500], np.int32)))
    short = run_decode(p, c, qs[1], kv=B.paged_kv(c.k_d, c.v_d, c.table_d, 32, c.n_pages))[0]
    q.copy_(qs[1])
    graph.replay()
    t.cuda.synchronize()
    assert t.equal(o, short) and (short[0] == 0).all()
