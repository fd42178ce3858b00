"""Attention of chunks of new tokens in a batch of many slots of which few have rows."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, normal
from tests.gpu_util import dev, torch
from tests.serving_util import check_chunk, host, offsets, run_chunk

pytestmark = pytest.mark.gpu


def compare(batch, new, lens, hq=4, hkv=1, seed=71):
    """new and lens: of the busy slots, {slot: number}; the others hold no tokens."""
    rng = np.random.default_rng(seed)
    all_lens, all_new = np.zeros(batch, np.int64), np.zeros(batch, np.int64)
    for n, w in new.items():
        all_lens[n], all_new[n] = lens[n], w
    c = Cache(rng, all_lens, hkv, 16)
    q, cu = normal(rng, int(all_new.sum()), hq, 128), offsets(all_new)
    print("[slots]", batch, new, flush=True)
    o, ls = run_chunk(B.ChunkProblem(batch, hq, hkv, c.width, q.shape[0]), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, all_lens, cu), int(all_lens.max()))


@pytest.mark.parametrize("batch", [2, 3, 64, 65, 66, 257, 258, 259, 322, 513, 1025, 2000])
def test_one_busy_slot_at_each_end(batch):
    compare(batch, {0: 3, batch - 1: 4}, {0: 200, batch - 1: 90})


@pytest.mark.parametrize("gap", [1, 2, 63, 64, 65, 255, 256, 257, 258, 320, 511, 512, 513, 1500])
def test_idle_slots_between_busy_ones(gap):
    """`gap` idle slots behind the first busy one, and another busy one right behind the second."""
    compare(gap + 300, {0: 2, gap + 1: 3, gap + 2: 1}, {0: 100, gap + 1: 60, gap + 2: 10}, 6, 2)


def test_slots_at_random():
    rng = np.random.default_rng(72)
    slots = sorted(rng.choice(4000, 40, replace=False))
    lens = {int(n): int(rng.integers(1, 80)) for n in slots}
    compare(4000, {n: int(rng.integers(1, x + 1)) for n, x in lens.items()}, lens, 3, 1)


def test_offsets_out_of_their_range_leave_slots_idle():
    """Offsets below 0 and behind n_rows are read as 0 and n_rows: such slots have no rows, and are passed over."""
    rng = np.random.default_rng(73)
    cu = np.concatenate([np.full(200, -5), [0, 0, 7], np.full(600, 7), [9, 9], np.full(100, 500)]).astype(np.int32)
    lens = np.zeros(len(cu) - 1, np.int64)
    lens[[199, 201, 802, 804]] = 30, 40, 50, 60
    c = Cache(rng, lens, 1, 16)
    q = normal(rng, 12, 4, 128)
    o, ls = run_chunk(B.ChunkProblem(len(lens), 4, 1, c.width, 12), c, dev(q), dev(cu))
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, lens, cu), 60)


def call_us(batch, busy):
    """One call in microseconds, the shortest of several runs of 20."""
    t = torch()
    rng = np.random.default_rng(74)
    lens, new = np.zeros(batch, np.int64), np.zeros(batch, np.int64)
    lens[busy], new[busy] = 1000, 4
    c = Cache(rng, lens, 1, 16)
    kv = c.upload()
    p = B.ChunkProblem(batch, 4, 1, c.width, int(new.sum()))
    q, cu, n = dev(normal(rng, p.n_rows, 4, 128)), dev(offsets(new)), B.cosa_chunk_workspace_bytes(p)
    ws, o = t.empty(n, dtype=t.uint8, device="cuda"), t.empty(p.n_rows, 4, 128, dtype=t.int16, device="cuda")
    best = float("inf")
    for _ in range(6):
        a, b = t.cuda.Event(enable_timing=True), t.cuda.Event(enable_timing=True)
        a.record()
        for _ in range(20):
            B.cosa_chunk_attention(p, q, kv, c.lens_d, cu, ws, n, o)
        b.record()
        t.cuda.synchronize()
        best = min(best, a.elapsed_time(b) / 20 * 1e3)
    return best


def test_idle_slots_are_not_walked_one_by_one():
    """8192 slots, two of them busy, side by side or at the two ends. One slot at a time, even at 100 ns a slot, would add 800 us to
    a call of some 30; the bound leaves a factor of more than two on either side."""
    side_by_side, ends = call_us(8192, [0, 1]), call_us(8192, [0, 8191])
    print(f"[slots] side by side {side_by_side:.1f} us, at the ends {ends:.1f} us", flush=True)
    assert ends < 4 * side_by_side + 100
