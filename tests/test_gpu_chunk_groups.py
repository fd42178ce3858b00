"""Attention of chunks of new tokens with odd numbers of rows in a unit, over several ranges: partial results have room for one
row more than a unit has, and end with the workspace."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, normal
from tests.gpu_util import dev, torch
from tests.serving_util import check_chunk, host, offsets

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,lens,new", [
    (1, 1, [3000], [1]), (3, 1, [5000, 700], [1, 0]), (3, 1, [4000, 300], [90, 200]), (10, 2, [2500, 900], [60, 1]),
    (11, 1, [6000], [3]), (17, 1, [3000], [33]), (129, 1, [2000], [2]), (257, 1, [1500], [2])])
def test_against_the_oracle_with_a_workspace_of_just_its_size(hq, hkv, lens, new):
    t = torch()
    rng = np.random.default_rng(81)
    c = Cache(rng, lens, hkv, 16)
    kv, cu = c.upload(), offsets(new)
    q = normal(rng, int(cu[-1]), hq, 128)
    p = B.ChunkProblem(len(lens), hq, hkv, c.width, q.shape[0])
    n, guard = B.cosa_chunk_workspace_bytes(p), 4096
    ws = t.full((n + 2 * guard,), 0xA5, dtype=t.uint8, device="cuda")
    o = t.full((q.shape[0], hq, 128), 0x7FC0, dtype=t.int16, device="cuda")
    ls = t.full((q.shape[0], hq), float("nan"), device="cuda")
    print("[groups]", hq, hkv, lens, new, flush=True)
    B.cosa_chunk_attention(p, dev(q), kv, c.lens_d, dev(cu), ws[guard:], n, o, ls)
    t.cuda.synchronize()
    assert (ws[:guard] == 0xA5).all() and (ws[guard + n:] == 0xA5).all()
    check_chunk(*host(o, ls), S.chunk_attention(q, c.k, c.v, c.table, lens, cu), max(lens))
