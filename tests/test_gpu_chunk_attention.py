"""Attention of chunks of new tokens over a paged cache against the float64 oracle."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, as_f64, normal, run_decode
from tests.gpu_util import dev, torch
from tests.serving_util import check_chunk, host, offsets, run_chunk

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)


def one(seed, hq, hkv, page, lens, new, lse=True, width=None, extra=0, sm_scale=0.0):
    rng = np.random.default_rng(seed)
    c = Cache(rng, lens, hkv, page, width=width)
    cu = offsets(new)
    q = normal(rng, int(cu[-1]) + extra, hq, 128)
    p = B.ChunkProblem(len(lens), hq, hkv, c.width, q.shape[0], sm_scale=sm_scale)
    say("[chunk]", seed, hq, hkv, page, lens, new)
    o, ls = run_chunk(p, c, dev(q), dev(cu), lse)
    ref = S.chunk_attention(q, c.k, c.v, c.table, lens, cu, sm_scale)
    check_chunk(*host(o, ls), ref, max(list(lens) + [1]))
    return p, c, q, cu, o, ls


@pytest.mark.parametrize("hq,hkv,page,lens,new", [
    (1, 1, 16, [1], [1]),
    (4, 1, 16, [5], [5]),
    (4, 1, 16, [1000], [16]),
    (4, 2, 32, [127], [127]),
    (4, 2, 32, [128], [128]),
    (4, 2, 32, [129], [129]),
    (8, 2, 64, [300, 0, 1, 64, 517], [300, 0, 1, 1, 200]),
    (7, 1, 16, [400, 37], [100, 37]),
    (12, 1, 128, [700], [45]),
    (20, 1, 256, [513, 256], [30, 13]),
    (5, 5, 16, [300, 260], [280, 1]),
    (128, 1, 64, [200], [5]),
    (256, 1, 64, [130], [3]),
    (300, 1, 16, [140], [3]),
    (6, 3, 1024, [1500], [1100]),
])
def test_against_the_oracle(hq, hkv, page, lens, new):
    one(1, hq, hkv, page, lens, new)


@pytest.mark.parametrize("seed", range(4))
def test_ragged_batches(seed):
    rng = np.random.default_rng(100 + seed)
    hkv = int(rng.choice([1, 2, 3]))
    g = int(rng.choice([1, 2, 3, 4, 7, 8]))
    lens = [int(x) for x in rng.integers(0, 900, 9)]
    new = [int(rng.integers(0, n + 1)) if rng.random() < 0.6 else min(n, 1) for n in lens]
    one(seed, g * hkv, hkv, int(rng.choice([16, 32, 64, 256])), lens, new, lse=seed % 2 == 0, extra=5)


def test_a_unit_over_many_ranges():
    """Few rows over a long context: a unit is cut into many ranges and joined."""
    one(2, 4, 1, 64, [20000], [3])
    one(3, 8, 2, 16, [9000, 4000], [70, 1])


def test_rows_in_front_of_token_0_see_nothing():
    """More rows than tokens: the first ones have no token (their positions are below 0)."""
    _, _, _, cu, o, ls = one(4, 4, 2, 16, [10, 0, 300], [200, 70, 310])
    assert (as_f64(o)[:190] == 0).all() and np.isneginf(ls.cpu().numpy()[:190]).all()
    assert (as_f64(o)[200:270] == 0).all()


@pytest.mark.parametrize("length", [256, 257, 2048, 2049, 8192, 8193])
def test_units_of_so_many_parts(length):
    """One unit in 1, 2, 8, 9, 32 and 33 ranges; its rows are shared out among their workgroups from 9 on."""
    one(5, 4, 1, 64, [length], [3])


def test_many_rows_of_many_parts():
    one(6, 4, 1, 32, [12000], [64])
    one(7, 10, 2, 32, [300, 7000], [2, 50])
    one(8, 300, 1, 16, [3000], [2])
