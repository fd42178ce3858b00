"""Attention of chunks of new tokens where it can go wrong: infinite and NaN values, extreme logits, malformed device
data, strides, large offsets, many sequences, streams and graphs."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from paper_2607_25291_amd.inputs import f32_to_bf16_bits
from tests.decode_util import Cache, as_f64, normal, run_decode
from tests.gpu_util import dev, torch
from tests.serving_util import check_chunk, host, offsets, run_chunk

pytestmark = pytest.mark.gpu

INF, NEG, NAN = np.uint16(0x7F80), np.uint16(0xFF80), np.uint16(0x7FC0)


def say(*a):
    print(*a, flush=True)


def check_odd(o, lse, ref, longest):
    """check_chunk for results with infinities and NaN: these equal the oracle's, the rest is held to its tolerance."""
    ro, rl, wt, mag = (x.copy() for x in ref)
    odd = ~np.isfinite(ro)
    assert np.array_equal(np.isnan(o), np.isnan(ro)) and (o[np.isinf(ro)] == ro[np.isinf(ro)]).all()
    bad = np.isnan(rl)
    assert np.array_equal(np.isnan(lse), bad)
    for x in (o, ro, wt):
        x[odd] = 0.0
    for x in (lse, rl, mag):
        x[bad] = 0.0
    check_chunk(o, lse, (ro, rl, np.where(np.isfinite(wt), wt, 0.0), np.where(np.isfinite(mag), mag, 0.0)), longest)


@pytest.mark.parametrize("hq,hkv,page,length,new", [(4, 1, 16, 300, 300), (2, 2, 32, 700, 150), (7, 1, 64, 400, 90)])
@pytest.mark.parametrize("where", ["v", "k"])
@pytest.mark.parametrize("values", [[INF], [NEG], [NAN], [INF, NEG, NAN]])
def test_infinite_and_nan_rows_reach_only_the_rows_that_see_them(hq, hkv, page, length, new, where, values):
    rng = np.random.default_rng(31)
    c = Cache(rng, [length], hkv, page)
    cu = offsets([new])
    q = normal(rng, new, hq, 128)
    first = length - new
    tokens = [first + 3, first + new // 2, length - 2] + ([first // 2] if first else [])
    for i, t in enumerate(tokens):
        (c.v if where == "v" else c.k)[c.table[0, t // page], i % hkv, t % page, 5 + 40 * i % 128] = values[i % len(values)]
    if where == "k":
        # q's sign decides between a logit of +inf and -inf: only NaN and -inf have a result that is a number
        q[..., :] = np.where(np.isin(q, [0, 0x8000]), np.uint16(0x3F80), q) & np.uint16(0x7FFF)
    p = B.ChunkProblem(1, hq, hkv, c.width, new)
    say("[odd]", hq, hkv, page, length, new, where, values)
    o, ls = run_chunk(p, c, dev(q), dev(cu))
    ref = S.chunk_attention(q, c.k, c.v, c.table, [length], cu)
    check_odd(*host(o, ls), ref, length)


def test_rows_whose_logits_are_all_minus_infinity():
    rng = np.random.default_rng(32)
    c = Cache(rng, [40, 200], 1, 16)
    q = normal(rng, 240, 4, 128) & np.uint16(0x7FFF)
    for t in range(20):
        c.k[c.table[0, t // 16], 0, t % 16, 3] = NEG
    cu = offsets([40, 200])
    o, ls = run_chunk(B.ChunkProblem(2, 4, 1, c.width, 240), c, dev(q), dev(cu))
    assert (as_f64(o)[:20] == 0).all() and np.isneginf(ls.cpu().numpy()[:20]).all()
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, [40, 200], cu), 200)


@pytest.mark.parametrize("size,sm_scale", [(1.0, 300.0), (2.0 ** 40, 0.0), (2.0 ** 60, 1e-16), (1.0, 3e38), (2.0 ** 16, 1.0)])
def test_extreme_logits(size, sm_scale):
    """The row's largest logit takes all the weight: the result is its value, whatever the logits' size."""
    rng = np.random.default_rng(33)
    c = Cache(rng, [260], 2, 16, sinks=False)
    q = f32_to_bf16_bits(size * rng.standard_normal((100, 4, 128), dtype=np.float32))
    p = B.ChunkProblem(1, 4, 2, c.width, 100, sm_scale=sm_scale)
    o, ls = run_chunk(p, c, dev(q), dev(offsets([100])))
    ref = S.chunk_attention(q, c.k, c.v, c.table, [260], offsets([100]), sm_scale)
    o, ls = host(o, ls)
    # rows whose second logit lies far enough below the first for any order of fp32 sums
    from oracle.cosa_oracle import default_scale, widen
    scale, clear = default_scale(128, sm_scale), np.zeros((100, 4), bool)
    at = np.arange(260)
    for h in range(4):
        k = widen(c.k[c.table[0, at // 16], h // 2, at % 16])
        for i in range(100):
            s = np.sort((k @ widen(q[i, h]))[:161 + i])
            big = (np.abs(k) @ np.abs(widen(q[i, h]))).max()
            clear[i, h] = (s[-1] - s[-2] - 2.0 ** -16 * big) * scale > 40
    assert clear.any()
    err = np.abs(o - ref[0])[clear]
    assert np.isfinite(o).all() and (err <= 2.0 ** -7 * np.abs(ref[0][clear]) + 1e-15).all()
    with np.errstate(over="ignore"):
        want = ref[1].astype(np.float32)
    fine = clear & np.isfinite(want)
    assert (np.abs(ls[fine] - ref[1][fine]) <= 2.0 ** -16 * ref[3][fine]).all()


def test_malformed_device_data():
    """Lengths, offsets and table entries outside their ranges are read as the header says; nothing else is written."""
    rng = np.random.default_rng(34)
    c = Cache(rng, [90, 40, 64], 2, 16, width=7)
    c.k[c.k == NAN], c.v[c.v == NAN] = 0, 0
    c.table[:, :][c.table == 2 ** 31 - 1] = -9
    q = normal(rng, 120, 6, 128)
    cases = [([90, 40, 64], [0, 50, 70, 110]), ([2 ** 31 - 1, -5, 64], [0, 50, 70, 110]), ([90, 40, 64], [-7, 30, 20, 500]),
             ([90, 40, 64], [0, 0, 0, 0]), ([90, 40, 64], [500, 600, 700, 800]), ([0, 0, 0], [0, 40, 80, 120]),
             ([90, 40, 64], [60, 30, 10, 120])]
    for lens, cu in cases:
        say("[malformed]", lens, cu)
        c.lens = np.asarray(lens, np.int32)
        cu = np.asarray(cu, np.int32)
        o, ls = run_chunk(B.ChunkProblem(3, 6, 2, 7, 120), c, dev(q), dev(cu))
        check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, lens, cu), 112)
    c.lens = np.asarray([90, 40, 64], np.int32)
    c.table[0, 2], c.table[2, 0] = c.n_pages, -2 ** 31
    cu = offsets([60, 10, 20])
    o, ls = run_chunk(B.ChunkProblem(3, 6, 2, 7, 120), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, c.lens, cu), 112)


def test_a_table_without_pages():
    rng = np.random.default_rng(35)
    c = Cache(rng, [0, 0], 1, 16, width=0)
    o, ls = run_chunk(B.ChunkProblem(2, 2, 1, 0, 5), c, dev(normal(rng, 5, 2, 128)), dev(offsets([2, 2])),
                      lens=dev(np.array([7, 0], np.int32)))
    o, ls = host(o, ls)
    assert (o[:4] == 0).all() and np.isneginf(ls[:4]).all() and np.isnan(o[4]).all() and np.isnan(ls[4]).all()


def test_strided_queries_and_streams():
    t = torch()
    rng = np.random.default_rng(36)
    c = Cache(rng, [333, 80], 2, 32)
    cu = dev(offsets([100, 33]))
    q = dev(normal(rng, 133, 8, 128))
    p = B.ChunkProblem(2, 8, 2, c.width, 133)
    o, ls = run_chunk(p, c, q, cu)
    wide = dev(normal(rng, 140, 12, 128))
    wide[:133, 2:10] = q
    side = t.cuda.Stream()
    t.cuda.synchronize()
    for stream in (None, side):
        o2, ls2 = run_chunk(p, c, wide[:, 2:10], cu, stream=stream)
        assert t.equal(o, o2) and t.equal(ls, ls2)
    with t.cuda.stream(side):
        o3, _ = run_chunk(p, c, q, cu, lse=False)
    assert t.equal(o, o3)


def test_one_token_equals_a_decode_step():
    """Sequences of one new token each: the decode call's result but for the bf16 weights."""
    rng = np.random.default_rng(37)
    lens = [1, 17, 900, 5000, 0]
    c = Cache(rng, lens, 2, 16)
    q = normal(rng, 5, 8, 128)
    kv = c.upload()
    o, ls = run_chunk(B.ChunkProblem(5, 8, 2, c.width, 5), c, dev(q), dev(offsets([1] * 5)), kv=kv)
    od, lsd = run_decode(B.DecodeProblem(5, 8, 2, c.width), c, dev(q), kv=kv)
    ref = S.chunk_attention(q, c.k, c.v, c.table, lens, offsets([1] * 5))
    check_chunk(*host(o, ls), ref, 5000)
    check_chunk(*host(od, lsd), ref, 5000)


def test_many_sequences():
    """More sequences than a workgroup has threads, most of them without rows."""
    rng = np.random.default_rng(38)
    n = 1700
    lens = rng.integers(0, 60, n)
    new = np.where(rng.random(n) < 0.1, rng.integers(0, 5, n), 0)
    new[-1] = 3
    c = Cache(rng, lens, 1, 16)
    q = normal(rng, int(new.sum()), 3, 128)
    cu = offsets(new)
    o, ls = run_chunk(B.ChunkProblem(n, 3, 1, c.width, q.shape[0]), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, lens, cu), 60)


def test_pages_behind_4_gib():
    t = torch()
    rng = np.random.default_rng(39)
    hkv, page, n_pages, length, new = 4, 256, 20000, 1000, 70
    gen = t.Generator(device="cuda").manual_seed(1)
    k = t.zeros(n_pages, hkv, page, 128, dtype=t.bfloat16, device="cuda")
    v = t.zeros_like(k)
    table = np.array([[19999, 17000, 3, 18888]], np.int32)
    for p in table[0]:
        for x in (k, v):
            x[int(p)] = t.randn(hkv, page, 128, generator=gen, device="cuda").to(t.bfloat16)
    q = normal(rng, new, 8, 128)
    pick = lambda x: x[t.from_numpy(table[0].astype(np.int64)).cuda()].view(t.int16).cpu().numpy().view(np.uint16)
    ref = S.chunk_attention(q, pick(k), pick(v), np.arange(4)[None], [length], offsets([new]))
    kv = B.paged_kv(k, v, dev(table), page, n_pages)
    c = Cache(rng, [length], hkv, page, width=4)
    keep = dev(table)
    kv = B.paged_kv(k, v, keep, page, n_pages)
    o, ls = run_chunk(B.ChunkProblem(1, 8, hkv, 4, new), c, dev(q), dev(offsets([new])), kv=kv,
                      lens=dev(np.array([length], np.int32)))
    check_chunk(*host(o, ls), ref, length)


def test_results_are_deterministic_and_workspaces_carry_nothing():
    t = torch()
    rng = np.random.default_rng(40)
    c = Cache(rng, [3000, 40, 900], 2, 16)
    cu = dev(offsets([200, 40, 1]))
    q = dev(normal(rng, 241, 8, 128))
    p = B.ChunkProblem(3, 8, 2, c.width, 241)
    kv = c.upload()
    n = B.cosa_chunk_workspace_bytes(p)
    ws = t.full((n,), 0xFF, dtype=t.uint8, device="cuda")
    first = None
    for i in range(4):
        o, ls = t.zeros(241, 8, 128, dtype=t.int16, device="cuda"), t.zeros(241, 8, device="cuda")
        lens = c.lens_d if i != 2 else dev(np.array([100, 0, 2], np.int32))
        B.cosa_chunk_attention(p, q, kv, lens, cu, ws, n, o, ls)
        t.cuda.synchronize()
        if first is None:
            first = (o, ls)
        elif i != 2:
            assert t.equal(o, first[0]) and t.equal(ls, first[1])


def test_captured_and_replayed():
    """Two graphs that share a workspace, replayed in turn while lengths and offsets change, with eager calls between."""
    t = torch()
    rng = np.random.default_rng(41)
    c = Cache(rng, [2000, 700, 64], 2, 16)
    kv = c.upload()
    p = B.ChunkProblem(3, 8, 2, c.width, 150)
    n = B.cosa_chunk_workspace_bytes(p)
    ws, ws2 = (t.full((n,), 0xFF, dtype=t.uint8, device="cuda") for _ in range(2))
    q = [dev(normal(rng, 150, 8, 128)) for _ in range(2)]
    lens, cu = dev(np.array([2000, 700, 64], np.int32)), dev(offsets([100, 49, 1]))
    o = [t.zeros(150, 8, 128, dtype=t.int16, device="cuda") for _ in range(3)]
    ls = [t.zeros(150, 8, device="cuda") for _ in range(3)]
    B.cosa_chunk_attention(p, q[0], kv, lens, cu, ws, n, o[0], ls[0])
    t.cuda.synchronize()
    graphs = []
    for i in range(2):
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            B.cosa_chunk_attention(p, q[i], kv, lens, cu, ws, n, o[i], ls[i])
        graphs.append(g)
    for step in range(6):
        new = [[100, 49, 1], [1, 1, 1], [0, 150, 0], [60, 0, 64], [149, 0, 1], [50, 50, 50]][step]
        cu.copy_(dev(offsets(new)))
        lens.copy_(dev(np.array([2000 - 300 * step, 700 - 100 * step, 64], np.int32)))
        for i in range(2):
            for x in (o[i], o[2]):
                x.zero_()
            for x in (ls[i], ls[2]):
                x.zero_()
            graphs[i].replay()
            B.cosa_chunk_attention(p, q[i], kv, lens, cu, ws2, n, o[2], ls[2])
            t.cuda.synchronize()
            assert t.equal(o[i], o[2]) and t.equal(ls[i], ls[2]), (step, i)


@pytest.mark.parametrize("batch", [63, 64, 65, 512, 513])
def test_batches_around_the_lanes_and_threads(batch):
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, 90, batch)
    new = np.where(rng.random(batch) < 0.5, np.minimum(lens, 1), rng.integers(0, 20, batch))
    new[0], new[-1] = 0, 7
    c = Cache(rng, lens, 2, 16)
    q = normal(rng, int(new.sum()), 6, 128)
    cu = offsets(new)
    say("[batch]", batch)
    o, ls = run_chunk(B.ChunkProblem(batch, 6, 2, c.width, q.shape[0]), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, lens, cu), 90)


def test_groups_over_several_units_of_several_kv_heads():
    rng = np.random.default_rng(42)
    c = Cache(rng, [300, 5], 2, 16)
    q, cu = normal(rng, 6, 1200, 128), offsets([5, 1])
    o, ls = run_chunk(B.ChunkProblem(2, 1200, 2, c.width, 6), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, [300, 5], cu), 300)


def test_pages_that_rows_share():
    """Forked sequences, and a page that one row holds twice."""
    rng = np.random.default_rng(43)
    c = Cache(rng, [200, 180, 0, 96], 2, 32)
    c.table[1, :5] = c.table[0, :5]
    c.table[2, :4], c.lens[2] = c.table[0, :4], 128
    c.table[3, 2] = c.table[3, 0]
    new = [40, 20, 128, 96]
    q, cu = normal(rng, sum(new), 4, 128), offsets(new)
    o, ls = run_chunk(B.ChunkProblem(4, 4, 2, c.width, sum(new)), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, c.lens, cu), 200)


def test_two_calls_at_once():
    """Two streams, each with its own workspace and outputs."""
    t = torch()
    rng = np.random.default_rng(44)
    c = Cache(rng, [4000, 900, 1, 333], 2, 16)
    kv = c.upload()
    streams = [t.cuda.Stream() for _ in range(2)]
    calls = []
    for new in ([500, 30, 1, 100], [1, 1, 1, 1]):
        p = B.ChunkProblem(4, 8, 2, c.width, sum(new))
        q, cu = dev(normal(rng, sum(new), 8, 128)), dev(offsets(new))
        n = B.cosa_chunk_workspace_bytes(p)
        calls.append((p, q, cu, run_chunk(p, c, q, cu, kv=kv), t.empty(n, dtype=t.uint8, device="cuda"), n,
                      t.zeros(sum(new), 8, 128, dtype=t.int16, device="cuda"), t.zeros(sum(new), 8, device="cuda")))
    t.cuda.synchronize()
    for _ in range(5):
        for s, (p, q, cu, _, ws, n, o, ls) in zip(streams, calls):
            B.cosa_chunk_attention(p, q, kv, c.lens_d, cu, ws, n, o, ls, stream=s)
    t.cuda.synchronize()
    for *_, want, ws, n, o, ls in calls:
        assert t.equal(o, want[0]) and t.equal(ls, want[1])
