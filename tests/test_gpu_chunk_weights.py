"""Attention of chunks of new tokens where an infinite value meets a weight of 0: its key's logit is -inf."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2607_25291_amd import binding as B
from tests.decode_util import Cache, normal
from tests.gpu_util import dev
from tests.serving_util import host, offsets, run_chunk
from tests.test_gpu_chunk_edges import INF, NAN, NEG, check_odd

pytestmark = pytest.mark.gpu


def positive(rng, *shape):
    q = normal(rng, *shape)
    return np.where(np.isin(q, [0, 0x8000]), np.uint16(0x3F80), q) & np.uint16(0x7FFF)


def compare(c, q, new, o, ls):
    """Magnitudes of the logits, for the tolerance, without the infinite ones: their keys have no weight."""
    cu, finite = offsets(new), np.where(c.k == NEG, np.uint16(0), c.k)
    o_ref, lse_ref, wt, _ = S.chunk_attention(q, c.k, c.v, c.table, c.lens, cu)
    mag = S.chunk_attention(q, finite, np.zeros_like(c.v), c.table, c.lens, cu)[3]
    assert np.isnan(o_ref).any() and np.isfinite(mag).all() and np.isfinite(lse_ref).all()
    check_odd(*host(o, ls), (o_ref, lse_ref, wt, mag), int(max(c.lens)))
    return o_ref


def case(lens, new, hq, hkv, page, keys, value, seed=61):
    """Sequence n: the tokens keys[n] have a key element of -inf, which queries of positive elements make a logit of
    -inf, and two value elements of `value`."""
    rng = np.random.default_rng(seed)
    c = Cache(rng, lens, hkv, page)
    q = positive(rng, sum(new), hq, 128)
    for n, tokens in enumerate(keys):
        for i, t in enumerate(tokens):
            at = c.table[n, t // page], slice(None), t % page
            c.k[at][:, (3 + 50 * i) % 128] = NEG
            c.v[at][:, (7 + 40 * i) % 128] = value
            c.v[at][:, (77 + 40 * i) % 128] = value
    print("[weight 0]", lens, new, hq, hkv, page, keys, flush=True)
    o, ls = run_chunk(B.ChunkProblem(len(lens), hq, hkv, c.width, sum(new)), c, dev(q), dev(offsets(new)))
    compare(c, q, new, o, ls)


@pytest.mark.parametrize("value", [INF, NEG, NAN])
@pytest.mark.parametrize("token", [5, 130, 270, 299])
def test_in_tiles_that_all_rows_see_and_in_those_at_the_edge(token, value):
    """300 tokens, the last 20 of them new: keys 0 to 255 lie in tiles that every row sees, the others in the edge tile."""
    case([300], [20], 4, 1, 16, [[token]], value)


@pytest.mark.parametrize("length", [255, 256, 257, 383, 384, 385, 400])
def test_the_length_of_the_context_does_not_matter(length):
    """The same key and value, the border of the tiles moves past it."""
    case([length], [2], 4, 1, 32, [[250]], INF)


def test_units_of_several_ranges():
    """Partial results that are joined, and whole units beside them."""
    case([9000, 4000, 140], [70, 1, 140], 8, 2, 16, [[10, 4600, 8940, 8999], [3990], [100, 139]], INF)


def test_beside_an_infinite_value_that_has_weight():
    """One token's infinity has a weight, another one's has none: NaN where they share an element, infinity elsewhere."""
    rng = np.random.default_rng(62)
    c = Cache(rng, [300], 1, 16)
    q = positive(rng, 30, 4, 128)
    for t, key in ((285, True), (290, False)):
        at = c.table[0, t // 16], 0, t % 16
        if key:
            c.k[at][9] = NEG
        c.v[at][20] = INF
        c.v[at][40 if key else 60] = INF
    o, ls = run_chunk(B.ChunkProblem(1, 4, 1, c.width, 30), c, dev(q), dev(offsets([30])))
    ref = compare(c, q, [30], o, ls)
    assert np.isnan(ref[20:, :, [20, 40]]).all() and np.isinf(ref[20:, :, 60]).all()


def test_rows_of_nothing_but_such_keys():
    """Every logit that a row sees is -inf: 0 and -inf, whatever the values are."""
    rng = np.random.default_rng(63)
    c = Cache(rng, [40], 1, 16)
    q = positive(rng, 40, 4, 128)
    for t in range(12):
        at = c.table[0, t // 16], 0, t % 16
        c.k[at][3], c.v[at][t] = NEG, INF
    o, ls = run_chunk(B.ChunkProblem(1, 4, 1, c.width, 40), c, dev(q), dev(offsets([40])))
    o, ls = host(o, ls)
    assert (o[:12] == 0).all() and np.isneginf(ls[:12]).all() and np.isnan(o[12:, :, :12]).all()
