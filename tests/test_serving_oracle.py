"""CPU pins of the serving oracle: independent routines, closed forms, examples by hand, and invariants of whole rounds."""
import numpy as np
import pytest
import torch

from oracle import decode_oracle as D
from oracle import serving_oracle as S
from oracle.cosa_oracle import widen
from paper_2607_25291_amd.inputs import f32_to_bf16_bits


def bits(rng, *shape):
    return f32_to_bf16_bits(rng.standard_normal(shape).astype(np.float32))


@pytest.mark.parametrize("lens,new", [([37], [37]), ([50, 33], [7, 1]), ([20, 64, 1], [20, 16, 1])])
def test_chunks_against_torch(lens, new):
    rng = np.random.default_rng(1)
    pages, page, hq, hkv = 16, 16, 4, 2
    k, v = bits(rng, pages, hkv, page, 128), bits(rng, pages, hkv, page, 128)
    table = rng.permutation(pages)[:4 * len(lens)].reshape(len(lens), 4)
    cu = np.concatenate([[0], np.cumsum(new)])
    q = bits(rng, cu[-1], hq, 128)
    o, lse, _, _ = S.chunk_attention(q, k, v, table, lens, cu)
    for n, (length, w) in enumerate(zip(lens, new)):
        at = np.arange(length)
        kk, vv = (torch.tensor(widen(x[table[n, at // page], :, at % page])).transpose(0, 1).repeat_interleave(2, 0) for x in (k, v))
        qq = torch.tensor(widen(q[cu[n]:cu[n + 1]])).transpose(0, 1)
        mask = torch.arange(length) <= torch.arange(length - w, length)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(qq, kk, vv, attn_mask=mask)
        assert np.abs(want.transpose(0, 1).numpy() - o[cu[n]:cu[n + 1]]).max() < 1e-6  # the scale is a fp32 number
        # one token is a decode step
        d, ds = D.decode_attention(q[cu[n + 1] - 1:cu[n + 1]], k, v, table[n:n + 1], [length])[:2]
        assert np.allclose(d[0], o[cu[n + 1] - 1], atol=1e-12) and np.allclose(ds[0], lse[cu[n + 1] - 1], atol=1e-12)


def test_chunk_closed_forms():
    # keys of 0: a row's result is the mean of the values it sees, its sum their number
    v = f32_to_bf16_bits(np.arange(64, dtype=np.float32).reshape(4, 1, 16, 1) * np.ones(128, np.float32))
    q = np.full((12, 1, 128), 0x3F80, np.uint16)
    o, lse, _, _ = S.chunk_attention(q, np.zeros_like(v), v, np.array([[0, 1, 2, 3], [0, 1, 2, 3]]), [40, 2], [0, 5, 10])
    for i in range(5):
        assert np.allclose(o[i], (35 + i) / 2) and np.allclose(lse[i], np.log(36 + i))
    assert (o[5:8] == 0).all() and np.isneginf(lse[5:8]).all()  # in front of token 0
    assert np.allclose(o[8], 0) and np.allclose(o[9], 0.5) and np.isnan(o[10:]).all()


def test_fork_by_hand():
    # page 16; row 0: 20 tokens (a page of 4), row 1: 32 (whole pages), row 2: 5
    table = np.array([[7, 3, -1], [4, 6, -1], [9, -1, -1]])
    old = np.full((6, 3), -5)
    t, lens, src, dst, rows = S.page_fork([0, 0, 1, 1, 2, 0], table, [20, 32, 5], 16, 0, [11, 12, 13], 3, old)
    assert t.tolist() == [[7, 3, -5], [7, 11, -5], [4, 6, -5], [4, 6, -5], [9, -5, -5], [7, 12, -5]]
    assert lens.tolist() == [20, 20, 32, 32, 5, 20]
    assert src.tolist() == [3, 3] and dst.tolist() == [11, 12] and rows.tolist() == [4, 4]
    t, lens, src, dst, rows = S.page_fork([0, 2, -1, 0], table, [20, 32, 5], 16, 1, [11, 12, 13], 2, old[:4])
    assert lens.tolist() == [20, 5, 0, 0] and t.tolist() == [[7, 11, -5], [12, -5, -5], [-5, -5, -5], [-5, -5, -5]]
    assert src.tolist() == [3, 9] and rows.tolist() == [4, 5]


def test_release_and_compact_by_hand():
    table = np.array([[7, 3, 1], [7, 6, -1]])
    # row 0 ends, row 1 keeps its first page: 1, 3 and 6 become free; 2 and 5 are left of the list
    assert S.page_release(table, [40, 30], table, [0, 10], 16, 10, [0, 2, 5], 3, 1) == [2, 5, 1, 3, 6]
    t, moves, free = S.page_compact(table, [40, 30], 16, 10, 9)
    assert moves == [(7, 0), (6, 2)] and free == [4, 5, 6, 7, 8, 9]
    assert t.tolist() == [[0, 3, 1], [0, 2, -1]]
    t, moves, free = S.page_compact(table, [40, 30], 16, 10, 1)
    assert moves == [(7, 0)] and free == [2, 4, 5, 7, 8, 9] and t.tolist() == [[0, 3, 1], [0, 6, -1]]


@pytest.mark.parametrize("seed", range(6))
def test_rounds_lose_no_page_and_no_token(seed):
    """Fork, copy, release and compact in turn: the pages are those held and those listed, each once, and every sequence
    keeps its tokens."""
    rng = np.random.default_rng(seed)
    page, n_pages, width, rows = 16, 60, 6, 5
    k = rng.integers(0, 65536, (n_pages, 1, page, 2)).astype(np.uint16)
    v = k.copy()
    lens = rng.integers(0, width * page + 1, rows)
    table, free = np.full((rows, width), -1), list(rng.permutation(n_pages))
    for r in range(rows):
        for j in range(-(-int(lens[r]) // page)):
            table[r, j] = free.pop()

    def tokens(table, lens):
        return [[k[table[r, t // page], 0, t % page].tolist() for t in range(lens[r])] for r in range(len(lens))]

    for _ in range(4):
        parent = rng.integers(-1, rows, rows)
        before = tokens(table, lens)
        t2, l2, src, dst, keep = S.page_fork(parent, table, lens, page, 0, free, len(free), np.full((rows, width), -1))
        S.page_copy(k, v, None, src, dst, keep, len(src))
        assert tokens(t2, l2) == [before[p] if p >= 0 else [] for p in parent]
        # a page that two rows hold is full in both: neither writes to it
        last = [(r, t2[r, l2[r] // page]) for r in range(rows) if l2[r] % page]
        for r, p in last:
            assert not any(p in t2[x, :-(-int(l2[x]) // page)] for x in range(rows) if x != r)
        free = S.page_release(table, lens, t2, l2, page, n_pages, free, len(free), len(src))
        table, lens = t2, l2
        used = {p for _, _, p in S.held(table, lens, page, n_pages)}
        assert sorted(free + list(used)) == list(range(n_pages))
        before = tokens(table, lens)
        table, moves, free = S.page_compact(table, lens, page, n_pages, 1000)
        s, d = np.array(moves, dtype=int).reshape(-1, 2).T
        S.page_copy(k, v, None, s, d, None, len(s))
        assert tokens(table, lens) == before
        assert {p for _, _, p in S.held(table, lens, page, n_pages)} == set(range(len(used)))
