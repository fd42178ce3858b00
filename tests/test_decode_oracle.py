"""CPU pins of the decode oracle: closed forms, brute force and independent routines."""
import math

import numpy as np
import pytest

from oracle import decode_oracle as D
from oracle.cosa_oracle import widen
from paper_2607_25291_amd.inputs import f32_to_bf16_bits


def test_page_map_by_hand():
    # page 16; request 0: 10 cached + 1 (fits its page), 1: 16 + 1 (takes a page), 2: 0 + 33 (takes three)
    table = np.array([[7, -1, -1], [3, -1, -1], [-1, -1, -1]])
    t, seq, cu, slots, taken = D.page_map([10, 16, 0], [1, 1, 33], [5, 9, 2, 4, 8], 5, table, 16, 40)
    assert t.tolist() == [[7, -1, -1], [3, 5, -1], [9, 2, 4]]
    assert seq.tolist() == [11, 17, 33] and cu.tolist() == [0, 1, 2, 35] and taken == 4
    assert slots[:3].tolist() == [7 * 16 + 10, 5 * 16, 9 * 16] and slots[34] == 4 * 16
    assert (slots[35:] == -1).all()
    # one page short: the last request adds nothing, the pages of the others stay
    t, seq, cu, slots, taken = D.page_map([10, 16, 0], [1, 1, 33], [5, 9, 2, 4, 8], 3, table, 16, 40)
    assert seq.tolist() == [11, 17, 0] and taken == 1 and (slots[2:] == -1).all()
    assert t[2].tolist() == [-1, -1, -1]


def test_bounds_hold_every_key():
    rng = np.random.default_rng(0)
    k = f32_to_bf16_bits(rng.standard_normal((40, 2, 128)).astype(np.float32))
    kc, vc = np.zeros((4, 2, 16, 128), np.uint16), np.zeros((4, 2, 16, 128), np.uint16)
    b = np.full((4, 2, 2, 128), 0x7FC0, np.uint16)
    slots = np.array([2 * 16 + i for i in range(16)] + [i for i in range(16)] + [3 * 16 + i for i in range(8)])
    D.kv_append(kc, vc, b, k, k, slots)
    for p, rows in ((2, slice(0, 16)), (0, slice(16, 32)), (3, slice(32, 40))):
        assert np.array_equal(widen(b[p, :, 0]), widen(k[rows]).min(0))
        assert np.array_equal(widen(b[p, :, 1]), widen(k[rows]).max(0))
    assert (b[1] == 0x7FC0).all()
    # the score bounds every logit
    q = f32_to_bf16_bits(rng.standard_normal((1, 4, 128)).astype(np.float32))
    table = np.array([[2, 0, 3]])
    s, _ = D.page_score(q, b, table, [40], 16)
    for h in range(4):
        logits = widen(k[:, h // 2]) @ widen(q[0, h]) * float(np.float32(1 / math.sqrt(128)))
        for j in range(3):
            assert s[0, h, j] >= logits[16 * j:16 * (j + 1)].max() - 1e-12


@pytest.mark.parametrize("p,args,want", [
    (10, (1.0, 1, 4, 1, 1), 4), (3, (1.0, 1, 8, 1, 1), 3), (100, (0.1, 1, 64, 0, 0), 10),
    (100, (0.1, 20, 64, 0, 0), 20), (100, (0.01, 1, 64, 3, 4), 7), (0, (1.0, 1, 4, 1, 1), 0),
])
def test_kept_pages(p, args, want):
    assert D.kept_pages(p, *args) == want


def test_selection_prefers_row_maxima_then_lower_index():
    score = np.array([[[5, 1, 3, 3, 0, 2], [0, 9, 1, 1, 8, 2]]], np.float32)
    pages, count = D.page_select(score, [6 * 16], 16, 1, 1.0, 1, 4, 0, 0)
    # differences: [0,-4,-2,-2,-5,-3] and [-9,0,-8,-8,-1,-7] -> maxima [0,0,-2,-2,-1,-3]
    assert pages[0, 0].tolist() == [0, 1, 2, 4] and count[0, 0] == 4
    pages, _ = D.page_select(score, [6 * 16 - 15], 16, 1, 1.0, 1, 3, 0, 1)
    assert pages[0, 0].tolist() == [0, 1, 5]


def test_attention_against_direct_softmax():
    rng = np.random.default_rng(1)
    x = lambda *s: f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32))
    q, kc, vc = x(2, 4, 128), x(9, 2, 16, 128), x(9, 2, 16, 128)
    table = np.array([[8, 1, 5], [0, 2, 7]])
    o, lse, _, _ = D.decode_attention(q, kc, vc, table, [41, 0])
    k = np.concatenate([widen(kc[p, 1]) for p in table[0]])[:41]
    v = np.concatenate([widen(vc[p, 1]) for p in table[0]])[:41]
    s = k @ widen(q[0, 3]) * float(np.float32(1 / math.sqrt(128)))
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(o[0, 3], w @ v, rtol=0, atol=1e-12)
    assert abs(lse[0, 3] - math.log(np.exp(s).sum())) < 1e-12
    assert (o[1] == 0).all() and np.isneginf(lse[1]).all()
    # the list of all pages, in another order, changes nothing; foreign entries add nothing
    pages = np.array([[[2, 0, 1, 3, -1]] * 2] * 2)
    o2, lse2, _, _ = D.decode_attention(q, kc, vc, table, [41, 0], pages, np.array([[5, 5], [2, 0]]))
    assert np.allclose(o2, o, atol=1e-12) and np.allclose(lse2[0], lse[0], atol=1e-12)
