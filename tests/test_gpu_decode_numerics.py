"""What the attention of one new token keeps of its weights and values: all 32 bits of a weight in the product with V,
and infinite values."""
import sys

import numpy as np
import pytest

from oracle import decode_oracle as D
from oracle.cosa_oracle import widen
from paper_2607_25291_amd import binding as B
from paper_2607_25291_amd.inputs import f32_to_bf16_bits
from tests.decode_util import Cache, as_f64, check_attention, normal, run_decode
from tests.gpu_util import dev

pytestmark = pytest.mark.gpu


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


def few_elements(rng, lens, hq, hkv, page, width):
    """A cache and queries whose logits are exact in fp32: queries of 1 and of a random number in [1, 2) in their first
    two elements, keys with those two elements only (0 here), values of 0."""
    c = Cache(rng, lens, hkv, page, width, sinks=False)
    q = np.zeros((len(lens), hq, 128), np.uint16)
    q[:, :, 0] = 0x3F80
    q[:, :, 1] = f32_to_bf16_bits(rng.uniform(1.0, 1.99, (len(lens), hq)).astype(np.float32))
    for x in (c.k, c.v):
        x[x != 0x7FC0] = 0
    return c, q


# lengths, heads, KV heads, page, table width: one workgroup a unit, split units, 32 columns a unit
SHAPES = {"whole": ([3, 33, 150], 4, 2, 16, 20), "split": ([3, 900, 2100], 4, 2, 16, 200),
          "columns_32": ([3 + 11 * i % 500 for i in range(260)], 20, 1, 16, 32), "columns_32_split": ([3, 4100, 900], 48, 2, 64, 400)}


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("name", list(SHAPES))
def test_weights_keep_32_bits(name, listed):
    """Tokens 1 and 2 of every sequence have logits -x and -x - 2^-12 q1 and values of opposite signs, token 0 a
    logit of 0 and the others -3, and no values: what is left is 2^-12 of a weight, where rounding both weights to
    16 bits leaves up to 2^-17.

    The logits are exact in fp32 (20 bits). A weight is exp2 of one fused product: the rounding of scale * log2(e),
    2^-24 of at most 3, is one factor of nearly equal size for both; its own is half a unit in the last place of a number
    below 4 (2^-23); exp2 has one unit (2^-23). So 2^-22 for each weight of the two, and fp32 sums of their products and
    the joins' powers of two with 2^-23 each time the two are scaled apart, which they are not in one tile: 2^-20 of
    their sum has room for all. The sum of all weights and the joins' common factors err relative to the result
    (longest / 128 + 548 terms of 2^-24: 2^-14), and the output is rounded to bf16: 2^-8 of itself."""
    lens, hq, hkv, page, width = SHAPES[name]
    say(f"[decode weights] {name} listed {listed}")
    rng = np.random.default_rng(len(name))
    c, q = few_elements(rng, lens, hq, hkv, page, width)
    for n, length in enumerate(lens):
        for j in range(-(-length // page)):
            c.k[c.table[n, j], :, :min(page, length - j * page), 0] = 0xC040  # -3
        at = c.table[n, 0]
        x = f32_to_bf16_bits(-rng.uniform(0.1, 1.9, hkv).astype(np.float32))
        c.k[at, :, 0, 0], c.k[at, :, 1, 0], c.k[at, :, 2, 0] = 0, x, x
        c.k[at, :, 2, 1] = 0xB980  # -2^-12
        v = f32_to_bf16_bits(rng.uniform(0.5, 2.0, (hkv, 128)).astype(np.float32))
        c.v[at, :, 1], c.v[at, :, 2] = v, v ^ 0x8000
    p = B.DecodeProblem(len(lens), hq, hkv, c.width, sm_scale=1.0)
    lists = None
    if listed:
        pages = np.tile(np.arange(c.width, dtype=np.int32), (len(lens), hkv, 1))
        lists = (pages, np.array([[-(-n // page)] * hkv for n in lens], np.int32))
    o, _ = run_decode(p, c, dev(q), lists, lse=False)
    ro, _, wt, _ = D.decode_attention(q, c.k, c.v, c.table, lens, sm_scale=1.0)
    assert (np.abs(ro) < 2.0 ** -11 * wt).all() and (ro != 0).all()
    err = np.abs(as_f64(o) - ro)
    tol = (2.0 ** -8 + 2.0 ** -14) * np.abs(ro) + 2.0 ** -20 * wt
    assert (err <= tol).all(), f"off by {err.max()}, worst ratio {(err / tol).max()}"


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("name", list(SHAPES))
def test_infinite_values(name, listed):
    """An infinite value with any weight down to 2^-92 of the largest gives that infinity in its element, one of either
    sign NaN; the other elements stay what they are. Logits of 0 to -64, one for each token (mod 65)."""
    lens, hq, hkv, page, width = SHAPES[name]
    say(f"[decode infinite values] {name} listed {listed}")
    rng = np.random.default_rng(len(name) + 7)
    c, q = few_elements(rng, lens, hq, hkv, page, width)
    for n, length in enumerate(lens):
        at = lambda i: (c.table[n, i // page], slice(None), i % page)
        for i in range(length):
            c.k[at(i)][:, 0] = f32_to_bf16_bits(np.array(-(i % 65), np.float32))
            c.v[at(i)] = f32_to_bf16_bits(rng.standard_normal((hkv, 128)).astype(np.float32))
        for h in range(hkv):
            for d in range(64):  # one token in elements 0 .. 31, two in 32 .. 63, of opposite signs from 48 on
                i, j = (int(x) for x in rng.integers(0, length, 2))
                i, j = (i, j) if d >= 4 else (0, 0)  # elements 0 .. 3: the token of largest weight
                sign = 0x8000 * int(rng.integers(0, 2))
                c.v[c.table[n, i // page], h, i % page, d] = 0x7F80 | sign
                if d >= 32 and i != j:
                    c.v[c.table[n, j // page], h, j % page, d] = 0x7F80 | (sign if d < 48 else 0x8000 - sign)
    p = B.DecodeProblem(len(lens), hq, hkv, c.width, sm_scale=1.0)
    lists = None
    if listed:
        pages = np.tile(np.arange(c.width, dtype=np.int32), (len(lens), hkv, 1))
        lists = (pages, np.array([[-(-n // page)] * hkv for n in lens], np.int32))
    o, lse = run_decode(p, c, dev(q), lists)
    with np.errstate(invalid="ignore"):
        ro, rl, wt, mag = D.decode_attention(q, c.k, c.v, c.table, lens, sm_scale=1.0)
    assert np.isinf(ro).any() and np.isnan(ro).any()
    got, odd = as_f64(o), ~np.isfinite(ro)
    assert np.array_equal(got[odd], ro[odd], equal_nan=True)
    wt[odd] = ro[odd] = got[odd] = 0
    check_attention(got, lse.cpu().numpy().astype(np.float64), (ro, rl, wt, mag), max(lens))


@pytest.mark.parametrize("listed", [False, True])
@pytest.mark.parametrize("scale", [1.0, 2.0 ** 60])
@pytest.mark.parametrize("name", list(SHAPES))
def test_large_logits(name, scale, listed):
    """Logits of +-2^33 (1 + j / 128), apart by 2^26 at least where they differ (and 2^60 times as large): only the tokens
    of the largest have weight, 1 each, in every head. o is the mean of at most three values: nine products of their
    weights' terms in fp32 (2^-24 of the magnitudes for each, 2^-20 with room), and a rounding to bf16 (2^-9 of it, taken
    as 2^-8 with the division). lse: the logit times the scale is exact, plus log(n) of at most log 3: half a unit of
    fp32, 2^-24 of it."""
    lens, hq, hkv, page, width = SHAPES[name]
    say(f"[decode large logits] {name} scale {scale} listed {listed}")
    rng = np.random.default_rng(len(name) + 3)
    c, q = few_elements(rng, lens, hq, hkv, page, width)
    q[:, :, 0] = 0x4980  # 2^20
    q[:, :, 1] = 0
    want, mag = np.zeros((2, len(lens), hq, 128))
    best = np.zeros((len(lens), hq))
    for n, length in enumerate(lens):
        sign = -1.0 if n % 2 else 1.0
        for h in range(hkv):
            j = rng.integers(0, 100, length)
            top = 100 if sign > 0 else -1
            at = rng.choice(length, int(rng.integers(1, 4)), replace=False)
            j[at] = top
            k = (sign * 2.0 ** 13 * (1 + (j + 1) / 128)).astype(np.float32)
            v = normal(rng, length, 128)
            i = np.arange(length)
            c.k[c.table[n, i // page], h, i % page, 0] = f32_to_bf16_bits(k)
            c.v[c.table[n, i // page], h, i % page] = v
            g = hq // hkv
            want[n, h * g:(h + 1) * g] = widen(v[at]).mean(0)
            mag[n, h * g:(h + 1) * g] = np.abs(widen(v[at])).mean(0)
            best[n, h * g:(h + 1) * g] = 2.0 ** 20 * float(k.max()) * scale + np.log(len(at))
            assert (widen(f32_to_bf16_bits(k)) == k).all() and (k == k.max()).sum() == len(at)
    p = B.DecodeProblem(len(lens), hq, hkv, c.width, sm_scale=scale)
    lists = None
    if listed:
        pages = np.tile(np.arange(c.width, dtype=np.int32), (len(lens), hkv, 1))
        lists = (pages, np.array([[-(-n // page)] * hkv for n in lens], np.int32))
    o, lse = run_decode(p, c, dev(q), lists)
    got = as_f64(o)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * mag).all()
    assert (np.abs(lse.cpu().numpy() - best) <= 2.0 ** -24 * np.abs(best)).all()


@pytest.mark.parametrize("name", list(SHAPES))
def test_largest_scale(name):
    """A scale whose product with log2(e) passes fp32: logits of 0 keep weight 1, any below them none; one or two tokens of
    0 per sequence, lse log(1) or log(2) (half a unit of fp32)."""
    lens, hq, hkv, page, width = SHAPES[name]
    say(f"[decode largest scale] {name}")
    rng = np.random.default_rng(len(name) + 5)
    c, q = few_elements(rng, lens, hq, hkv, page, width)
    want = np.zeros((len(lens), hq, 128))
    count = np.array([1 + n % 2 for n in range(len(lens))])
    for n, length in enumerate(lens):
        i = np.arange(length)
        at = rng.choice(length, count[n], replace=False)
        k = -rng.uniform(1e-6, 1.0, length).astype(np.float32)
        k[at] = 0
        v = normal(rng, length, 128)
        v[at] = v[at[:1]]
        c.k[c.table[n, i // page], :, i % page, 0] = f32_to_bf16_bits(k)[:, None]
        c.v[c.table[n, i // page], :, i % page] = v[:, None]
        want[n] = widen(v[at[0]])
    o, lse = run_decode(B.DecodeProblem(len(lens), hq, hkv, c.width, sm_scale=3e38), c, dev(q))
    # the same value once or twice over as many: exact but for the order of its three terms' products (2^-22), one rounding
    assert (np.abs(as_f64(o) - want) <= (2.0 ** -8 + 2.0 ** -22) * np.abs(want)).all()
    assert (np.abs(lse.cpu().numpy() - np.log(count)[:, None]) <= 2.0 ** -23).all()
