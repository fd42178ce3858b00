"""The decode-side operators together, as a serving program runs them: prompts enter the cache through
the page map, then decode steps add a token to every sequence and attend to all pages or to selected ones;
eagerly and as one captured step."""
import sys

import numpy as np
import pytest

from oracle import cosa_oracle as O
from oracle import decode_oracle as D
from paper_2607_25291_amd import binding as B
from paper_2607_25291_amd.inputs import random_inputs
from tests.decode_util import as_f64, check_attention, normal
from tests.gpu_util import dev, host_bits, torch

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


class Server:
    """Device state of a batch: cache, bounds, table, lengths and free list."""

    def __init__(self, batch, hq, hkv, page, width, n_pages, rows, seed):
        t = torch()
        z = lambda *s, dt=t.int32, fill=0: t.full(s, fill, dtype=dt, device="cuda")
        self.hq, self.hkv, self.page, self.n_pages, self.batch = hq, hkv, page, n_pages, batch
        self.kc = z(n_pages, hkv, page, 128, dt=t.int16, fill=0x7FC0)
        self.vc = self.kc.clone()
        self.bounds = z(n_pages, hkv, 2, 128, dt=t.int16, fill=0x7FC0)
        self.table = z(batch, width, fill=-1)
        self.cached, self.lens, self.new = z(batch), z(batch), z(batch)
        self.cu, self.taken = z(batch + 1), z(1)
        self.slots = z(rows, dt=t.int64)
        self.free = dev(np.random.default_rng(seed).permutation(n_pages).astype(np.int32))
        self.n_free = z(1, fill=n_pages)
        self.p = B.DecodeProblem(batch, hq, hkv, width)
        self.kv = B.paged_kv(self.kc, self.vc, self.table, page, n_pages)

    def add(self, k, v):
        """Maps and appends the packed rows; new holds how many each sequence adds. On the device throughout."""
        t = torch()
        self.cached.copy_(self.lens)
        B.cosa_page_map(self.batch, self.page, self.table.shape[1], self.cached, self.new, self.free, self.n_pages,
                        self.n_free, self.table, self.lens, self.cu, self.slots, self.slots.numel(), self.taken)
        B.cosa_kv_append(self.hkv, 128, self.page, self.n_pages, self.kc, self.vc, self.bounds, k.shape[0], k, v, self.slots)
        # the pages taken leave the front of the free list
        at = t.arange(self.n_pages, device="cuda") + self.taken
        self.free.copy_(self.free[at.clamp_max(self.n_pages - 1)])
        self.n_free.sub_(self.taken)

    def host(self):
        return (host_bits(self.kc), host_bits(self.vc), self.table.cpu().numpy(), self.lens.cpu().numpy())


def test_prompts_then_steps():
    t = torch()
    rng = np.random.default_rng(21)
    prompts, hq, hkv, page = [300, 0, 1, 64, 517], 8, 2, 32
    s = Server(5, hq, hkv, page, 20, 60, sum(prompts), 1)
    k, v = normal(rng, sum(prompts), hkv, 128), normal(rng, sum(prompts), hkv, 128)
    s.new.copy_(dev(np.array(prompts, np.int32)))
    s.add(dev(k), dev(v))
    want = [(k[a:a + n], v[a:a + n]) for a, n in zip(np.cumsum([0] + prompts), prompts)]
    budget = B.page_budget(6, sink_pages=1, recent_pages=2)
    n_ws = max(B.cosa_decode_workspace_bytes(s.p), B.cosa_decode_sparse_workspace_bytes(s.p, budget))
    ws = t.full((n_ws,), 0xFF, dtype=t.uint8, device="cuda")
    for step in range(34):  # past a page's end for every sequence
        k, v, q = normal(rng, 5, hkv, 128), normal(rng, 5, hkv, 128), normal(rng, 5, hq, 128)
        s.new.fill_(1)
        s.add(dev(k), dev(v))
        want = [(np.concatenate([a, k[i:i + 1]]), np.concatenate([b, v[i:i + 1]])) for i, (a, b) in enumerate(want)]
        if step not in (0, 1, 15, 33):
            continue
        say(f"[steps] {step}")
        kc, vc, table, lens = s.host()
        assert lens.tolist() == [len(a) for a, _ in want]
        bounds = host_bits(s.bounds)
        for i, (a, b) in enumerate(want):
            at = np.arange(len(a))
            assert np.array_equal(kc[table[i, at // page], :, at % page], a)
            assert np.array_equal(vc[table[i, at // page], :, at % page], b)
            for j in range(-(-len(a) // page)):
                rows = D.ordered(a[j * page:(j + 1) * page])
                assert np.array_equal(D.ordered(bounds[table[i, j], :, 0]), rows.min(0))
                assert np.array_equal(D.ordered(bounds[table[i, j], :, 1]), rows.max(0))
        used = table[table >= 0]
        assert len(set(used.tolist())) == len(used) == sum(-(-len(a) // page) for a, _ in want)

        o = t.zeros((5, hq, 128), dtype=t.int16, device="cuda")
        lse = t.zeros((5, hq), device="cuda")
        B.cosa_decode_attention(s.p, dev(q), s.kv, s.lens, ws, n_ws, o, lse)
        ref = D.decode_attention(q, kc, vc, table, lens)
        check_attention(as_f64(o), lse.cpu().numpy().astype(np.float64), ref, int(lens.max()))

        # selected pages: the three calls, then the one call, bit for bit; then against the oracle's attention
        score = t.zeros((5, hq, 20), device="cuda")
        pages = t.zeros((5, hkv, 6), dtype=t.int32, device="cuda")
        count = t.zeros((5, hkv), dtype=t.int32, device="cuda")
        o2, lse2 = t.zeros_like(o), t.zeros_like(lse)
        B.cosa_page_score(s.p, dev(q), s.kv, s.bounds, s.lens, score)
        B.cosa_page_select(s.p, page, s.lens, score, budget, pages, count)
        B.cosa_decode_attention_listed(s.p, dev(q), s.kv, s.lens, pages, count, 6, ws, n_ws, o2, lse2)
        o3, lse3 = t.zeros_like(o), t.zeros_like(lse)
        B.cosa_decode_sparse(s.p, dev(q), s.kv, s.bounds, s.lens, budget, ws, n_ws, o3, lse3)
        lay = B.cosa_decode_sparse_workspace_layout(s.p, budget)
        t.cuda.synchronize()
        assert t.equal(o2, o3) and t.equal(lse2, lse3)
        assert t.equal(ws[lay.pages:lay.pages + pages.numel() * 4].view(t.int32).view(pages.shape), pages)
        assert t.equal(ws[lay.count:lay.count + count.numel() * 4].view(t.int32).view(count.shape), count)
        want_pages, want_count = D.page_select(score.cpu().numpy(), lens, page, hkv, 1.0, 1, 6, 1, 2)
        assert np.array_equal(pages.cpu().numpy(), want_pages) and np.array_equal(count.cpu().numpy(), want_count)
        ref = D.decode_attention(q, kc, vc, table, lens, want_pages, want_count)
        check_attention(as_f64(o3), lse3.cpu().numpy().astype(np.float64), ref, 6 * page)


def test_captured_step():
    """One graph of a whole step (map, append, sparse and full attention), replayed step after step with
    the program's own eager work between the replays, against the same steps made eagerly."""
    t = torch()
    rng = np.random.default_rng(22)
    hq, hkv, page = 16, 2, 16
    budget = B.page_budget(5, sink_pages=1, recent_pages=1)
    prompts = [90, 200, 3]
    sides = []
    k0, v0 = normal(rng, sum(prompts), hkv, 128), normal(rng, sum(prompts), hkv, 128)
    for _ in range(2):
        s = Server(3, hq, hkv, page, 24, 80, sum(prompts), 2)
        s.new.copy_(dev(np.array(prompts, np.int32)))
        s.add(dev(k0), dev(v0))
        s.new.fill_(1)
        s.k, s.v = (t.zeros((3, hkv, 128), dtype=t.int16, device="cuda") for _ in range(2))
        s.q = t.zeros((3, hq, 128), dtype=t.int16, device="cuda")
        s.n_ws = B.cosa_decode_sparse_workspace_bytes(s.p, budget)
        s.ws = t.zeros(s.n_ws, dtype=t.uint8, device="cuda")
        s.o, s.o_all = t.zeros_like(s.q), t.zeros_like(s.q)
        sides.append(s)

    def step(s):
        s.add(s.k, s.v)
        B.cosa_decode_sparse(s.p, s.q, s.kv, s.bounds, s.lens, budget, s.ws, s.n_ws, s.o)
        B.cosa_decode_attention(s.p, s.q, s.kv, s.lens, s.ws, s.n_ws, s.o_all)

    eager, graphed = sides
    B.cosa_decode_sparse(eager.p, eager.q, eager.kv, eager.bounds, eager.lens, budget, eager.ws, eager.n_ws, eager.o)
    B.cosa_decode_attention(eager.p, eager.q, eager.kv, eager.lens, eager.ws, eager.n_ws, eager.o_all)
    t.cuda.synchronize()
    graph = t.cuda.CUDAGraph()
    with t.cuda.graph(graph):
        step(graphed)
    for i in range(40):
        k, v, q = (dev(normal(rng, 3, h, 128)) for h in (hkv, hkv, hq))
        for s in sides:
            for a, b in ((s.k, k), (s.v, v), (s.q, q)):
                a.copy_(b)
        step(eager)
        graph.replay()
        t.cuda.synchronize()
        for name in ("lens", "table", "slots", "taken", "bounds", "kc", "o", "o_all"):
            assert t.equal(getattr(eager, name), getattr(graphed, name)), (i, name)
    assert eager.lens.tolist() == [n + 40 for n in prompts]


def test_prefill_then_decode_reads_the_same_cache():
    """A prompt prefilled by cosa_prefill_paged from the cache that cosa_kv_append filled; the last prompt token as a
    decode query over that cache equals the oracle's dense attention in its row."""
    t = torch()
    L, hq, hkv, page = 512, 4, 2, 64
    q, k, v = random_inputs(1, hq, hkv, L, 128, seed=3)
    s = Server(1, hq, hkv, page, L // page, L // page + 2, L, 4)
    s.new.fill_(L)
    rows = lambda x: dev(np.ascontiguousarray(x[0].transpose(1, 0, 2)))
    s.add(rows(k), rows(v))
    prob = B.Problem(1, hq, hkv, L, 128, 128, 16)
    n = B.cosa_prefill_workspace_bytes(prob)
    ws = t.zeros(n, dtype=t.uint8, device="cuda")
    o = t.zeros((1, hq, L, 128), dtype=t.int16, device="cuda")
    B.cosa_prefill_paged(prob, dev(q), s.kv, B.select(B.SELECT_ALL), None, ws, n, o)
    last = t.zeros((1, hq, 128), dtype=t.int16, device="cuda")
    nd = B.cosa_decode_workspace_bytes(s.p)
    wd = t.zeros(nd, dtype=t.uint8, device="cuda")
    q_last = np.ascontiguousarray(q[:, :, -1])
    B.cosa_decode_attention(s.p, dev(q_last), s.kv, s.lens, wd, nd, last)
    kc, vc, table, lens = s.host()
    ref = D.decode_attention(q_last, kc, vc, table, lens)
    check_attention(as_f64(last), None, ref, L)
    dense = O.dense_attention(q, k, v, block=128)
    assert np.abs(ref[0][0] - dense[0, :, -1]).max() <= 1e-9
    # the prefill keeps its probabilities in bf16 (2^-8 each) and rounds its output once more
    assert (np.abs(as_f64(o)[0, :, -1] - ref[0][0]) <= 2.0 ** -8 * (np.abs(ref[0][0]) + ref[2][0]) + 2.0 ** -12).all()
