"""The serving operators together, as a serving program runs them: prompts enter in chunks, are sampled several times,
drafted tokens are verified and turned down, rows end, and the cache is compacted; eagerly and as captured steps."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.decode_util import normal
from tests.gpu_util import dev, host_bits, torch
from tests.serving_util import check_chunk, host

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


class Server:
    """Device state of a batch with two sets of tables and free lists, used in turn."""

    def __init__(self, batch, hq, hkv, page, width, n_pages, rows, seed):
        t = torch()
        z = lambda *s, dt=t.int32, fill=0: t.full(s, fill, dtype=dt, device="cuda")
        self.batch, self.hq, self.hkv, self.page, self.width, self.n_pages, self.rows = batch, hq, hkv, page, width, n_pages, rows
        self.kc = z(n_pages, hkv, page, 128, dt=t.int16, fill=0x7FC0)
        self.vc = self.kc.clone()
        self.bounds = z(n_pages, hkv, 2, 128, dt=t.int16, fill=0x7FC0)
        self.tables = [z(batch, width, fill=-1) for _ in range(2)]
        self.lens = [z(batch) for _ in range(2)]
        self.free = [dev(np.random.default_rng(seed).permutation(n_pages).astype(np.int32)), z(n_pages)]
        self.n_free = z(1, fill=n_pages)
        self.now, self.list = 0, 0
        self.cached, self.new, self.cu, self.taken = z(batch), z(batch), z(batch + 1), z(1)
        self.slots = z(rows, dt=t.int64)
        self.src, self.dst, self.part, self.parent = z(n_pages), z(n_pages), z(batch), z(batch)
        self.q = z(rows, hq, 128, dt=t.int16)
        self.k, self.v = z(rows, hkv, 128, dt=t.int16), z(rows, hkv, 128, dt=t.int16)
        self.o, self.lse = z(rows, hq, 128, dt=t.int16, fill=0x7FC0), z(rows, hq, dt=t.float32)
        self.p = B.ChunkProblem(batch, hq, hkv, width, rows)
        self.n_ws = max(B.cosa_chunk_workspace_bytes(self.p), B.cosa_page_workspace_bytes(n_pages))
        self.ws = t.full((self.n_ws,), 0xFF, dtype=t.uint8, device="cuda")

    @property
    def table(self):
        return self.tables[self.now]

    @property
    def length(self):
        return self.lens[self.now]

    def settle(self, old_table, old_lens, taken):
        """Pages that nobody holds any more go back; the pages taken leave the list."""
        B.cosa_page_release(self.page, self.width, self.n_pages, self.batch, old_table, old_lens, self.batch, self.table,
                            self.length, self.free[self.list], self.n_pages, self.n_free, taken, self.free[self.list ^ 1],
                            self.n_pages, self.n_free, self.ws, self.n_ws)
        self.list ^= 1

    def step(self):
        """The new tokens of every row (self.new; q, k and v packed) enter the cache and are attended to."""
        self.cached.copy_(self.length)
        B.cosa_page_map(self.batch, self.page, self.width, self.cached, self.new, self.free[self.list], self.n_pages,
                        self.n_free, self.table, self.length, self.cu, self.slots, self.rows, self.taken)
        B.cosa_kv_append(self.hkv, 128, self.page, self.n_pages, self.kc, self.vc, self.bounds, self.rows, self.k, self.v,
                         self.slots)
        kv = B.paged_kv(self.kc, self.vc, self.table, self.page, self.n_pages)
        B.cosa_chunk_attention(self.p, self.q, kv, self.length, self.cu, self.ws, self.n_ws, self.o, self.lse)
        self.settle(self.table, self.length, self.taken)

    def fork(self):
        """Rows go on as self.parent says."""
        was = self.now
        self.now ^= 1
        B.cosa_page_fork(self.batch, self.batch, self.page, self.width, self.parent, self.tables[was], self.lens[was], 0,
                         self.free[self.list], self.n_pages, self.n_free, self.table, self.length, self.src, self.dst,
                         self.part, self.taken)
        B.cosa_page_copy(self.hkv, 128, self.page, self.n_pages, self.kc, self.vc, self.bounds, self.src, self.dst, self.part,
                         self.batch, self.taken)
        self.settle(self.tables[was], self.lens[was], self.taken)

    def cut(self, lens):
        """Rows get shorter, or end."""
        self.cached.copy_(self.length)
        self.length.copy_(dev(np.asarray(lens, np.int32)))
        self.settle(self.table, self.cached, None)

    def compact(self, most):
        B.cosa_page_compact(self.batch, self.page, self.width, self.n_pages, self.table, self.length, most, self.table,
                            self.src, self.dst, self.taken, self.free[self.list], self.n_pages, self.n_free, self.ws, self.n_ws)
        B.cosa_page_copy(self.hkv, 128, self.page, self.n_pages, self.kc, self.vc, self.bounds, self.src, self.dst, None, most,
                         self.taken)


def check(s, want, fed=None):
    """Every row's tokens are in its pages; used and free pages are all the pages; the attention equals the oracle's."""
    t = torch()
    t.cuda.synchronize()
    kc, vc, table, lens = host_bits(s.kc), host_bits(s.vc), s.table.cpu().numpy(), s.length.cpu().numpy()
    assert lens.tolist() == [len(a) for a, _ in want]
    used = set()
    for i, (a, b) in enumerate(want):
        at = np.arange(len(a))
        assert np.array_equal(kc[table[i, at // s.page], :, at % s.page], a)
        assert np.array_equal(vc[table[i, at // s.page], :, at % s.page], b)
        pages = table[i, :-(-len(a) // s.page)].tolist()
        if len(a) % s.page:  # nobody else holds a page that will be written to
            assert all(pages[-1] not in table[r, :-(-len(want[r][0]) // s.page)] for r in range(s.batch) if r != i)
        used |= set(pages)
    n_free = int(s.n_free.item())
    free = s.free[s.list].cpu().numpy()[:n_free].tolist()
    assert len(set(free)) == n_free and not used & set(free) and used | set(free) == set(range(s.n_pages))
    if fed is not None:
        q, cu = fed
        o, lse = host(s.o, s.lse)
        rows = int(cu[-1])
        ref = S.chunk_attention(q[:rows], kc, vc, table, lens, cu)
        check_chunk(o[:rows], lse[:rows], ref, max(lens.tolist() + [1]))


def feed(s, rng, want, new):
    """Random rows for `new` tokens of every sequence, and the rows' tokens afterwards."""
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q, k, v = (normal(rng, s.rows, h, 128) for h in (s.hq, s.hkv, s.hkv))
    for a, b in ((s.q, q), (s.k, k), (s.v, v), (s.new, np.asarray(new, np.int32))):
        a.copy_(dev(b))
    out = [(np.concatenate([a, k[cu[i]:cu[i + 1]]]), np.concatenate([b, v[cu[i]:cu[i + 1]]])) for i, (a, b) in enumerate(want)]
    return out, (q, cu)


def test_chunks_samples_drafts_and_compaction():
    rng = np.random.default_rng(51)
    hkv = 2
    s = Server(6, 8, hkv, 16, 40, 150, 300, 1)
    want = [(np.zeros((0, hkv, 128), np.uint16),) * 2 for _ in range(6)]
    for new in ([100, 0, 40, 0, 0, 1], [100, 0, 1, 0, 0, 33], [57, 0, 1, 0, 0, 1]):  # prompts in chunks, beside single tokens
        want, fed = feed(s, rng, want, new)
        s.step()
        check(s, want, fed)
    parent = [0, 0, 0, 2, 5, 5]  # three samples of a prompt, two of another one, one row that moves
    s.parent.copy_(dev(np.array(parent, np.int32)))
    s.fork()
    want = [want[p] for p in parent]
    check(s, want)
    for step in range(3):
        want, fed = feed(s, rng, want, [5] * 6)  # five drafted tokens each ...
        s.step()
        check(s, want, fed)
        keep = [len(a) - int(rng.integers(0, 5)) for a, _ in want]  # ... of which some are turned down
        s.cut(keep)
        want = [(a[:n], b[:n]) for (a, b), n in zip(want, keep)]
        check(s, want)
    ends = [0 if i in (1, 4) else len(a) for i, (a, _) in enumerate(want)]
    s.cut(ends)
    want = [(a[:n], b[:n]) for (a, b), n in zip(want, ends)]
    check(s, want)
    s.compact(3)
    check(s, want)
    s.compact(s.n_pages)
    check(s, want)
    used = {int(p) for i, (a, _) in enumerate(want) for p in s.table.cpu().numpy()[i, :-(-len(a) // 16)]}
    assert used == set(range(len(used)))
    want, fed = feed(s, rng, want, [3, 20, 1, 1, 0, 40])
    s.step()
    check(s, want, fed)


def test_captured_rounds():
    """A step and a fork, captured once for each of the two tables, replayed in turn while lengths and parents change,
    against the same rounds made eagerly."""
    t = torch()
    rng = np.random.default_rng(52)
    sides = [Server(4, 4, 2, 16, 30, 120, 60, 2) for _ in range(2)]
    eager, graphed = sides
    prompts = [50, 3, 0, 7]

    def load(new, parent):
        for s in sides:
            s.new.copy_(dev(np.asarray(new, np.int32)))
            s.parent.copy_(dev(np.asarray(parent, np.int32)))
        q, k, v = (dev(normal(rng, 60, h, 128)) for h in (4, 2, 2))
        for s in sides:
            for a, b in ((s.q, q), (s.k, k), (s.v, v)):
                a.copy_(b)

    def round_(s):
        s.step()
        s.fork()

    load(prompts, [0, 1, 2, 3])
    for s in sides:
        round_(s)
    t.cuda.synchronize()
    graphs = []
    for _ in range(2):  # recorded, not run: the host's view of which table is the current one moves on
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            round_(graphed)
        graphs.append(g)
    for i in range(8):
        new = [[1, 1, 1, 1], [9, 0, 2, 1], [0, 0, 0, 0], [16, 16, 16, 12]][i % 4]
        parent = [[0, 0, 2, 3], [3, 1, 1, 0], [0, 1, 2, -1], [2, 2, 2, 2]][i // 2 % 4]
        load(new, parent)
        round_(eager)
        graphs[i % 2].replay()
        t.cuda.synchronize()
        # the eager side has moved its tables and lists along; the graphs hold theirs
        now, lst = eager.now, eager.list
        for name, a, b in (("table", eager.tables[now], graphed.tables[now]), ("lens", eager.lens[now], graphed.lens[now]),
                           ("free", eager.free[lst], graphed.free[lst]), ("n_free", eager.n_free, graphed.n_free),
                           ("k", eager.kc, graphed.kc), ("o", eager.o, graphed.o), ("bounds", eager.bounds, graphed.bounds)):
            assert t.equal(a, b), (i, name)
        say("[round]", i, eager.lens[now].tolist(), int(eager.n_free.item()))
