"""Attention of chunks of new tokens where slots need 64 bits: wide tables, lines past 2^31 slots, sequences close to
2^31 tokens."""
import numpy as np
import pytest

from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, as_f64, normal
from tests.gpu_util import dev, torch
from tests.serving_util import offsets, run_chunk

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,page,batch", [(8, 2, 16, 9), (5, 1, 32, 70), (300, 1, 16, 3)])
def test_the_width_of_a_table_changes_nothing(hq, hkv, page, batch):
    rng = np.random.default_rng(51)
    lens = [int(x) for x in rng.integers(0, 900, batch)]
    new = [int(rng.integers(0, x + 1)) if i % 3 else min(x, 1) for i, x in enumerate(lens)]
    c = Cache(rng, lens, hkv, page)
    n_rows = sum(new)
    q, cu = dev(normal(rng, n_rows, hq, 128)), dev(offsets(new))
    print("[wide]", hq, hkv, page, batch, flush=True)
    narrow = run_chunk(B.ChunkProblem(batch, hq, hkv, c.width, n_rows), c, q, cu)
    table = torch().zeros((batch, 1 << 20), dtype=torch().int32, device="cuda")
    table[:, :c.width] = c.table_d
    kv = B.paged_kv(c.k_d, c.v_d, table, page, c.n_pages)
    wide = run_chunk(B.ChunkProblem(batch, hq, hkv, 1 << 20, n_rows), c, q, cu, kv=kv)
    assert torch().equal(narrow[0], wide[0]) and torch().equal(narrow[1], wide[1])


def peaks(pages, page, rows):
    """Caches of zeros but for rows (page, row, element): logit 40 and value 1 in that element, for queries of `queries`.
    Every other key has weight e^-40."""
    t = torch()
    k, v = (t.zeros((pages, 1, page, 128), dtype=t.bfloat16, device="cuda") for _ in range(2))
    for p, row, d in rows:
        k[p, 0, row, 0] = 5.0
        v[p, 0, row, d] = 1.0
    return k.view(t.int16), v.view(t.int16)


def queries(n_rows, hq):
    t = torch()
    q = t.zeros((n_rows, hq, 128), dtype=t.bfloat16, device="cuda")
    q[..., 0] = 8.0
    return q.view(t.int16)


def check(o, lse, counts):
    """o [rows, Hq, 128]: element d has counts[row, d] keys of weight 1 (2^-8 for a weight's bf16, 2^-8 for the result's)."""
    total = counts.sum(1)
    want = (counts / total[:, None])[:, None, :]
    assert (np.abs(as_f64(o) - want) <= 2.0 ** -7 * want + 1e-7).all()
    assert (np.abs(lse.cpu().numpy() - (40 + np.log(total))[:, None]) <= 2.0 ** -15).all()


def test_a_line_past_2_31_slots():
    t, page, tokens, new, hq = torch(), 128, 1 << 22, 1024, 64
    table = np.zeros((1, tokens // page), np.int32)
    at = [i * 2048 + 37 * i % 2048 for i in range(16)] + [(tokens - 512) // page]  # the last one: for half of the rows
    for i, j in enumerate(at):
        table[0, j] = i + 1
    k, v = peaks(18, page, [(i + 1, 0, i + 7) for i in range(17)])
    entries = dev(table)  # the struct holds addresses
    kv = B.paged_kv(k, v, entries, page, 18)
    print("[line]", flush=True)
    o, ls = run_chunk(B.ChunkProblem(1, hq, 1, table.shape[1], new, sm_scale=1.0), None, queries(new, hq),
                      dev(offsets([new])), kv=kv, lens=t.tensor([tokens], dtype=t.int32, device="cuda"))
    counts = np.zeros((new, 128))
    counts[:, 7:23] = 1
    counts[new - 512:, 23] = 1
    check(o, ls, counts)


def test_sequences_of_almost_2_31_tokens():
    t, page, width, hq = torch(), 1 << 20, 2047, 4
    table = np.zeros((2, width), np.int32)
    table[0, [0, 1000, 2046]] = 1
    table[1, 2046] = 1
    lens, new = [width * page - 1, (width - 1) * page + 2], [1, 3]  # the second one's last rows see its last page's first row
    k, v = peaks(2, page, [(1, 0, 9), (1, page - 1, 100)])
    entries = dev(table)
    kv = B.paged_kv(k, v, entries, page, 2)
    print("[long]", flush=True)
    o, ls = run_chunk(B.ChunkProblem(2, hq, 1, width, 4, sm_scale=1.0), None, queries(4, hq), dev(offsets(new)), kv=kv,
                      lens=t.tensor(lens, dtype=t.int32, device="cuda"))
    counts = np.zeros((4, 128))
    counts[0, [9, 100]] = 3, 2
    counts[2:, 9] = 1
    rows = [0, 2, 3]
    check(o[rows], ls[rows], counts[rows])
    # row 1 stands in front of that page: 2^31 - 2^21 keys of logit 0
    assert (as_f64(o[1]) == 0).all()
    assert (np.abs(ls[1].cpu().numpy() - np.log((width - 1) * float(page))) <= 2.0 ** -15).all()  # sums of ones: exact below 2^24 in a range
