"""Pages of a cache forked, copied, released and compacted, against the oracle: whole numbers and copied bits, all equal."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.gpu_util import dev, host_bits, torch

pytestmark = pytest.mark.gpu

MARK = -77  # in every place that a call does not write


def say(*a):
    print(*a, flush=True)


def i32(x):
    return dev(np.asarray(x, np.int32))


def marked(*shape):
    return torch().full(shape, MARK, dtype=torch().int32, device="cuda")


class Rows:
    """A table of rows with random pages, some of which share the leading full pages of the row in front."""

    def __init__(self, rng, lens, page, width=None, spare=9, share=0.4):
        self.lens, self.page = np.asarray(lens, np.int32), page
        pages = [-(-int(n) // page) for n in lens]
        self.width = max(pages + [1]) if width is None else width
        self.table = np.full((len(lens), self.width), 2 ** 31 - 1, np.int32)
        need = max(sum(pages) + spare, 1)  # a cache has a page
        perm = rng.permutation(need).astype(np.int32)
        at = 0
        for r, p in enumerate(pages):
            k = 0
            if r and rng.random() < share:
                k = int(rng.integers(0, min(int(lens[r]), int(lens[r - 1])) // page + 1))
                self.table[r, :k] = self.table[r - 1, :k]
            self.table[r, k:p] = perm[at:at + p - k]
            at += p - k
        self.free, self.n_pages = perm[at:].copy(), need


def lengths(rng, n, longest, page):
    out = rng.integers(0, longest + 1, n)
    out[rng.random(n) < 0.2] = 0
    whole = rng.random(n) < 0.2
    out[whole] = out[whole] // page * page
    return out


def fork(t, parent, copy_all=0, n_free=None, free=None):
    n, w = len(parent), t.width
    free = t.free if free is None else np.asarray(free, np.int32)
    n_free = len(free) if n_free is None else n_free
    new, lens, src, dst, rows, taken = marked(n, w), marked(n), marked(n), marked(n), marked(n), marked(1)
    say("[fork]", len(t.lens), n, t.page, w, copy_all, n_free)
    B.cosa_page_fork(len(t.lens), n, t.page, w, i32(parent), i32(t.table), i32(t.lens), copy_all, i32(free), len(free),
                     i32([n_free]), new, lens, src, dst, rows, taken)
    got = [x.cpu().numpy() for x in (new, lens, src, dst, rows, taken)]
    want = S.page_fork(parent, t.table, t.lens, t.page, copy_all, free, n_free, np.full((n, w), MARK))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    k = len(want[2])
    assert got[5][0] == k
    for a, b in zip(got[2:5], want[2:]):
        assert np.array_equal(a[:k], b) and (a[k:] == MARK).all()
    return got


@pytest.mark.parametrize("rows,children,page,longest", [
    (1, 1, 16, 5), (1, 8, 64, 8001), (3, 0, 16, 100), (7, 30, 16, 3000), (300, 700, 32, 500), (40, 8192, 16, 90),
    (8192, 300, 128, 400), (2, 5, 1 << 20, 3 << 20)])
@pytest.mark.parametrize("copy_all", [0, 1])
def test_fork(rows, children, page, longest, copy_all):
    rng = np.random.default_rng(rows + children)
    t = Rows(rng, lengths(rng, rows, longest, page), page, spare=children + 3)
    parent = rng.integers(0, rows, children)
    parent[rng.random(children) < 0.1] = -1
    fork(t, parent, copy_all)


def test_fork_without_pages_left():
    rng = np.random.default_rng(5)
    t = Rows(rng, [33, 64, 5, 100], 16, spare=4)
    parent = [0, 0, 0, 1, 1, 2, 2, 3, 3, 0, 1, 2]
    for n_free in (0, 1, 3, 4, 100, -5):
        for copy_all in (0, 1):
            fork(t, parent, copy_all, n_free)
    fork(t, parent, 0, 0, free=[])
    fork(t, [0, 7, 4, -1, -2 ** 31, 2 ** 31 - 1])
    t.lens = np.array([-3, 2 ** 31 - 1, 5, 100], np.int32)  # read as clamped: a full row is not partly filled
    fork(t, parent)
    empty = Rows(rng, [], 16, width=3)
    fork(empty, [0, 1, -1])


@pytest.mark.parametrize("hkv,page,pairs,rows,bounds", [
    (1, 16, 1, False, True), (1, 16, 1, True, True), (3, 16, 40, True, True), (8, 64, 70, False, True), (8, 64, 33, True, False),
    (5, 256, 9, True, True), (2, 1024, 3, True, False), (70, 16, 4, True, True)])
def test_copy(hkv, page, pairs, rows, bounds):
    rng = np.random.default_rng(pairs + page)
    n_pages = 2 * pairs + 3
    bits = lambda *s: rng.integers(0, 2 ** 16, s, dtype=np.uint16)
    k, v = bits(n_pages, hkv, page, 128), bits(n_pages, hkv, page, 128)
    b = bits(n_pages, hkv, 2, 128) if bounds else None
    perm = rng.permutation(n_pages)
    src, dst = perm[:pairs].copy(), perm[pairs:2 * pairs].copy()
    if pairs > 3:  # pages outside the cache: skipped
        src[1], dst[2] = -1, n_pages
    r = rng.integers(-2, page + 3, pairs) if rows else None
    for n in sorted({pairs, pairs // 2, pairs + 5, 0, -1}):
        say("[copy]", hkv, page, pairs, n)
        kd, vd, bd = dev(k), dev(v), dev(b) if bounds else None
        B.cosa_page_copy(hkv, 128, page, n_pages, kd, vd, bd, i32(src), i32(dst), i32(r) if rows else None, pairs, i32([n]))
        want = [k.copy(), v.copy(), b.copy() if bounds else None]
        S.page_copy(*want, src, dst, r, n)
        for got, w in zip((kd, vd, bd), want):
            if w is not None:
                assert np.array_equal(host_bits(got), w)


def release(old, new, page, n_pages, free, n_free, n_taken, out_capacity=None, alias=False):
    (ot, ol), (nt, nl) = old, new
    cap = n_pages if out_capacity is None else out_capacity
    out, n_out = marked(max(cap, 1))[:cap], marked(1)
    n_ws = B.cosa_page_workspace_bytes(n_pages)
    ws = torch().full((n_ws,), 0xFF, dtype=torch().uint8, device="cuda")
    nf = i32([n_free])
    say("[release]", ot.shape, nt.shape, page, n_pages, len(free), n_free, n_taken, cap)
    same = nt is ot
    od = i32(ot)
    B.cosa_page_release(page, ot.shape[1], n_pages, ot.shape[0], od, i32(ol), nt.shape[0], od if same else i32(nt), i32(nl),
                        i32(free), len(free), nf, None if n_taken is None else i32([n_taken]), out, cap,
                        nf if alias else n_out, ws, n_ws)
    want = S.page_release(ot, ol, nt, nl, page, n_pages, free, n_free, n_taken or 0)
    k = min(len(want), cap)
    got = out.cpu().numpy()
    assert int((nf if alias else n_out).item()) == k
    assert got[:k].tolist() == want[:k] and (got[k:] == MARK).all()
    return got[:k]


@pytest.mark.parametrize("rows,page,longest,n_taken,alias", [
    (1, 16, 40, 0, False), (20, 16, 3000, 5, True), (64, 64, 20000, None, False), (300, 16, 9000, 40, False),
    (3, 1 << 18, 2 << 18, 1, True), (900, 16, 3000, 1, True)])
def test_release(rows, page, longest, n_taken, alias):
    """Rows that end, rows that get shorter, on both sides of the size for one workgroup."""
    rng = np.random.default_rng(rows)
    t = Rows(rng, lengths(rng, rows, longest, page), page, spare=50)
    new = np.where(rng.random(rows) < 0.3, 0, np.where(rng.random(rows) < 0.2, t.lens // 2, t.lens))
    release((t.table, t.lens), (t.table, new), page, t.n_pages, t.free, len(t.free), n_taken, alias=alias)
    release((t.table, t.lens), (t.table, t.lens), page, t.n_pages, t.free, len(t.free), n_taken)
    release((t.table, t.lens), (t.table, 0 * t.lens), page, t.n_pages, t.free, len(t.free), n_taken)


def test_release_edges():
    rng = np.random.default_rng(9)
    t = Rows(rng, [40, 0, 100, 33], 16, spare=6)
    zero = np.zeros(4, np.int32)
    old, gone = (t.table, t.lens), (t.table, zero)
    for n_free, n_taken in ((0, 0), (6, 6), (6, 9), (6, -1), (-4, 3), (50, 2), (3, 1)):
        release(old, gone, 16, t.n_pages, t.free, n_free, n_taken)
    for cap in (0, 1, 5, 9):
        release(old, gone, 16, t.n_pages, t.free, 6, 2, out_capacity=cap)
    release(old, gone, 16, t.n_pages, np.zeros(0, np.int32), 0, 0)
    # what the list has already is not added again; entries outside the cache are kept, and are no pages
    listed = np.array([int(t.table[0, 0]), -5, 2 ** 31 - 1, int(t.table[2, 1])], np.int32)
    release(old, gone, 16, t.n_pages, listed, 4, 0)
    release(old, gone, 16, t.n_pages, listed, 4, 1)
    bad = t.table.copy()
    bad[0, 1], bad[2, 0] = -1, t.n_pages
    release((bad, t.lens), (bad, zero), 16, t.n_pages, t.free, 6, 0)
    release((t.table[:0], zero[:0]), gone, 16, t.n_pages, t.free, 6, 3)
    release(old, (t.table[:0], zero[:0]), 16, t.n_pages, t.free, 6, 3)
    release((t.table, np.array([-1, 2 ** 31 - 1, 5, 5])), (t.table, np.array([0, 16, 5, -9])), 16, t.n_pages, t.free, 6, 3)


def compact(t, max_moves=None, lens=None, n_pages=None, in_place=False, capacity=None):
    n_pages = t.n_pages if n_pages is None else n_pages
    lens = t.lens if lens is None else lens
    most = n_pages if max_moves is None else max_moves
    cap = n_pages if capacity is None else capacity
    table = i32(t.table)
    new = table if in_place else torch().full_like(table, MARK)
    src, dst, free = (marked(max(x, 1))[:x] for x in (most, most, cap))
    n_moves, n_free = marked(1), marked(1)
    n_ws = B.cosa_page_workspace_bytes(n_pages)
    ws = torch().full((n_ws,), 0xFF, dtype=torch().uint8, device="cuda")
    say("[compact]", t.table.shape, t.page, n_pages, most, cap)
    B.cosa_page_compact(len(lens), t.page, t.width, n_pages, table, i32(lens), most, new, src, dst, n_moves, free, cap, n_free,
                        ws, n_ws)
    want, moves, unused = S.page_compact(t.table, lens, t.page, n_pages, most)
    k, f = len(moves), min(len(unused), cap)
    assert int(n_moves.item()) == k and int(n_free.item()) == f
    assert np.array_equal(new.cpu().numpy(), want)
    for got, w in ((src, [s for s, _ in moves]), (dst, [d for _, d in moves]), (free, unused[:f])):
        got = got.cpu().numpy()
        assert got[:len(w)].tolist() == w and (got[len(w):] == MARK).all()
    return new, moves


@pytest.mark.parametrize("rows,page,longest,spare", [
    (1, 16, 5, 0), (1, 16, 40, 30), (20, 16, 3000, 2000), (64, 64, 20000, 300), (300, 16, 9000, 5), (300, 16, 9000, 90000),
    (900, 16, 3000, 150000), (5, 16, 400, 4096 - 40)])
def test_compact(rows, page, longest, spare):
    rng = np.random.default_rng(rows + spare)
    t = Rows(rng, lengths(rng, rows, longest, page), page, spare=spare)
    full = compact(t)[1]
    compact(t, in_place=True)
    for most in (0, 1, len(full) // 2, len(full), len(full) + 1):
        compact(t, max_moves=most)


def test_compact_edges():
    rng = np.random.default_rng(6)
    t = Rows(rng, [100, 3, 0, 64], 16, spare=20)
    compact(t, capacity=0)
    compact(t, capacity=7)
    compact(t, lens=np.zeros(4, np.int32))
    compact(t, lens=np.array([-4, 2 ** 31 - 1, 0, 5], np.int32))
    compact(t, n_pages=11)  # entries outside the cache stay as they are
    for n in (4095, 4096, 4097, 8192, 40000):  # the last block of marks full, or not
        t = Rows(rng, rng.integers(0, 60000, 40), 16, spare=3, width=3750)
        if t.n_pages < n:
            t.n_pages = n
        compact(t)
    whole = Rows(rng, [16 * 4096], 16, spare=0)  # everything in use, whole blocks
    compact(whole)
    compact(Rows(rng, [], 16, width=2), n_pages=5)


@pytest.mark.parametrize("rows,longest", [(40, 900), (200, 14000)])
def test_release_from_one_table_and_from_two(rows, longest):
    """One table is read once, whichever length is the larger one; rows share pages, also within themselves."""
    rng = np.random.default_rng(rows)
    t = Rows(rng, lengths(rng, rows, longest, 16), 16, spare=50)
    table = t.table.copy()
    behind = np.arange(t.width)[None] >= -(-t.lens // 16)[:, None]
    table[behind] = rng.integers(0, t.n_pages, behind.sum())
    cap = t.width * 16
    pick = rng.integers(0, 4, rows)
    new = np.choose(pick, [np.zeros(rows, int), t.lens // 3, t.lens, np.minimum(t.lens + rng.integers(1, 500, rows), cap)])
    free = t.free[:30]
    one = release((table, t.lens), (table, new), 16, t.n_pages, free, len(free), 3)
    two = release((table, t.lens), (table.copy(), new), 16, t.n_pages, free, len(free), 3)
    assert np.array_equal(one, two)


def test_the_largest_pool():
    """Page numbers up to 2^28, lists shorter than what there is."""
    t, n_pages, cap = torch(), 1 << 28, 3000
    table = np.array([[n_pages - 1, 5, n_pages - 1 - 4096], [1 << 27, 0, 77], [n_pages // 3, 2, 1]], np.int32)
    lens = np.array([48, 33, 10], np.int32)
    used = {n_pages - 1, 5, n_pages - 1 - 4096, 1 << 27, 0, 77, n_pages // 3}
    n_ws = B.cosa_page_workspace_bytes(n_pages)
    ws = t.full((n_ws,), 0xFF, dtype=t.uint8, device="cuda")
    new, src, dst, n_moves, free, n_free = marked(3, 3), marked(4), marked(4), marked(1), marked(cap), marked(1)
    say("[largest]")
    B.cosa_page_compact(3, 16, 3, n_pages, i32(table), i32(lens), 4, new, src, dst, n_moves, free, cap, n_free, ws, n_ws)
    moves = list(zip(sorted(used)[:-5:-1], [1, 2, 3, 4]))
    assert list(zip(src.tolist(), dst.tolist())) == moves and n_moves.item() == 4
    to = dict(moves)
    want = [[to.get(int(p), int(p)) if j < -(-int(n) // 16) else int(p) for j, p in enumerate(row)] for row, n in zip(table, lens)]
    assert new.tolist() == want
    now = {to.get(p, p) for p in used}
    assert n_free.item() == cap and free.tolist() == [p for p in range(cap + 10) if p not in now][:cap]
    out, n_out = marked(9), marked(1)
    B.cosa_page_release(16, 3, n_pages, 3, i32(table), i32(lens), 1, i32(table[:1]), i32(lens[:1]), i32([n_pages - 2]), 1, i32([1]),
                        None, out, 9, n_out, ws, n_ws)
    assert n_out.item() == 5 and out.tolist() == [n_pages - 2, 0, 77, n_pages // 3, 1 << 27] + [MARK] * 4


def test_copy_behind_4_gib():
    t, n_pages, hkv, page = torch(), 20000, 4, 256
    k, v = (t.zeros((n_pages, hkv, page, 128), dtype=t.int16, device="cuda") for _ in range(2))
    for i, p in enumerate((19999, 3, 17001)):
        k[p], v[p] = i + 1, -i - 1
    say("[copy]", "4 GiB")
    B.cosa_page_copy(hkv, 128, page, n_pages, k, v, None, i32([19999, 3, 17001]), i32([18000, 19000, 0]), i32([256, 9, 100]), 3, i32([3]))
    for i, (d, keep) in enumerate(((18000, 256), (19000, 9), (0, 100))):
        for x, sign in ((k, 1), (v, -1)):
            assert (x[d, :, :keep] == sign * (i + 1)).all() and (x[d, :, keep:] == 0).all()
    assert (k.view(-1, hkv * page * 128)[:, 0] != 0).sum().item() == 6
