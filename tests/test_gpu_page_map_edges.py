"""Page maps at the ends of their range: a step without requests."""
import numpy as np
import pytest

from paper_2607_25291_amd import binding as B
from tests.gpu_util import torch

pytestmark = pytest.mark.gpu


def outputs(rows, fill=7):
    t = torch()
    z = lambda n, dt: t.full((n,), fill, dtype=dt, device="cuda")
    return z(3, t.int32), z(rows + 3, t.int64), z(2, t.int32)


@pytest.mark.parametrize("rows", [0, 1, 511, 513, 70000])
def test_an_empty_batch_leaves_nothing_of_the_step_before(rows):
    """No request: no row has a slot and no page is taken, whatever the outputs held; nothing behind them changes."""
    print(f"[page map] no requests, {rows} rows", flush=True)
    t = torch()
    cu, slots, taken = outputs(rows)
    B.cosa_page_map(0, 16, 8, None, None, None, 0, None, None, None, cu, slots, rows, taken)
    t.cuda.synchronize()
    assert cu.tolist() == [0, 7, 7] and taken.tolist() == [0, 7]
    assert (slots[:rows] == -1).all() and (slots[rows:] == 7).all()
    # each output by itself, the others left out; inputs that an empty batch does not use
    for keep in range(3):
        out = outputs(rows)
        a = [x if i == keep else None for i, x in enumerate(out)]
        free = t.arange(5, dtype=t.int32, device="cuda")
        B.cosa_page_map(0, 16, 8, None, None, free, 5, None, None, None, a[0], a[1], rows, a[2])
        t.cuda.synchronize()
        assert cu.tolist() == [0, 7, 7]
        for i, (x, want) in enumerate(zip(out, (cu, slots, taken))):
            assert t.equal(x, want) if i == keep else (x == 7).all()


def test_an_empty_step_between_others_in_a_captured_append():
    """A captured map and append, replayed: the graph of an empty batch clears the slots, so the append behind it writes
    nothing, though the step before filled the same buffers."""
    t = torch()
    rng = np.random.default_rng(0)
    i32 = lambda x: t.tensor(x, dtype=t.int32, device="cuda")
    page, rows = 16, 24
    kc, vc = (t.zeros((4, 1, page, 128), dtype=t.int16, device="cuda") for _ in range(2))
    table, lens, cu, taken = i32([[-1, -1]]), i32([0]), i32([0, 0]), i32([0])
    slots = t.zeros(rows, dtype=t.int64, device="cuda")
    free, n_free = i32([2, 1, 3, 0]), i32([4])
    k = t.from_numpy(rng.integers(1, 2 ** 14, (rows, 1, 128)).astype(np.int16)).cuda()

    def step(batch):
        B.cosa_page_map(batch, page, 2, i_cached, i_new, free, 4, n_free, table, lens, cu, slots, rows, taken)
        B.cosa_kv_append(1, 128, page, 4, kc, vc, None, rows, k, k, slots)
    i_cached, i_new = i32([0]), i32([20])
    graphs = []
    for batch in (1, 0):
        g = t.cuda.CUDAGraph()
        with t.cuda.graph(g):
            step(batch)
        graphs.append(g)
    for turn in range(3):
        graphs[0].replay()
        t.cuda.synchronize()
        assert taken.item() == 2 and (slots[:20] >= 0).all() and (slots[20:] == -1).all()
        assert t.equal(kc[2, 0], k[:16, 0]) and t.equal(vc[1, 0, :4], k[16:20, 0])
        kc.zero_()
        vc.zero_()
        graphs[1].replay()
        t.cuda.synchronize()
        assert taken.item() == 0 and cu[0].item() == 0 and (slots == -1).all()
        assert not kc.any() and not vc.any()


def test_rows_that_end_at_the_largest_number_of_rows():
    """2^31 - 1 rows: a request whose rows end there fits; one that would start there adds nothing, although the prefix
    sums stop at the same number."""
    t = torch()
    most = 2 ** 31 - 1
    i32 = lambda x: t.tensor(x, dtype=t.int32, device="cuda")
    print(f"[page map] {most} rows", flush=True)
    slots = t.zeros(most, dtype=t.int64, device="cuda")
    for new, lens, taken, last in (([most, 5], [0, 0], 0, [-1] * 3), ([most - 3, 3, 1], [0, 3, 0], 1, [48, 49, 50])):
        n = len(new)
        table, seq, cu = i32([[-7, -7]] * n), i32([-7] * n), i32([-7] * (n + 1))
        count = i32([-7])
        B.cosa_page_map(n, 16, 2, i32([0] * n), i32(new), i32([3, 1, 2]), 3, i32([3]), table, seq, cu, slots, most, count)
        t.cuda.synchronize()
        assert seq.tolist() == lens and count.item() == taken
        assert cu.tolist() == [0] + [min(sum(new[:i + 1]), most) for i in range(n)]
        assert table.tolist() == [[3 if x else -7, -7] for x in lens]
        assert slots[-3:].tolist() == last
        for a in range(0, most - 3, 2 ** 28):
            assert (slots[a:min(a + 2 ** 28, most - 3)] == -1).all()
