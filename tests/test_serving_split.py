"""The arithmetic that deals out an attention call over chunks (csrc/chunk_split.h), compiled for the host."""
import ctypes
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_25291_amd", "csrc")

SOURCE = r"""
#include "chunk_split.h"
using cosa::ChunkSeq;
extern "C" {
int chunk_rows() { return cosa::kChunkRows; }
int heads(int G) { return cosa::chunk_heads(G); }
int parts(int G) { return cosa::chunk_parts(G); }
int tokens(int G) { return cosa::chunk_tokens(G); }
ChunkSeq of(int len, int w, int G) { return {len, w, cosa::chunk_tokens(G), cosa::chunk_heads(G)}; }
int units(int len, int w, int G) { return of(len, w, G).units(); }
int keys(int len, int w, int G, int j) { return of(len, w, G).keys(j); }
int tiles(int len, int w, int G, int j) { return of(len, w, G).tiles(j); }
int key_slots(int len, int w, int G, int j) { return of(len, w, G).key_slots(j); }
int64_t start(int len, int w, int G, int j) { return of(len, w, G).start<int64_t>(j); }
int64_t slots(int len, int w, int G) { return of(len, w, G).slots<int64_t>(); }
// the unit that holds slot x, in rounds as the kernel's lanes search for it
int find(int len, int w, int G, int64_t x) {
  const ChunkSeq s = of(len, w, G);
  const int n = s.units();
  int first = 0;
  for (int step = cosa::search_step(n); step; step /= 64) {
    int hits = 0;
    for (int lane = 0; lane < 64; ++lane) {
      const int64_t i = (int64_t)first + (int64_t)lane * step;
      hits += i < n && s.start<int64_t>((int)i) <= x;
    }
    first += (hits - 1) * step;
  }
  return first;
}
int64_t range_length(int64_t total, int log2_most, int shortest) { return cosa::chunk_range<int64_t>(total, log2_most, shortest); }
int tile0(int64_t a, int64_t u, int key_slots) { return cosa::chunk_tile0<int64_t>(a, u, key_slots); }
int tile1(int64_t b, int64_t u, int key_slots, int tiles) { return cosa::chunk_tile1<int64_t>(b, u, key_slots, tiles); }
// where 31 bits are said to hold everything, they give the same
int narrow(long long batch, long long rows, long long cap, long long heads, int G) {
  return cosa::chunk_narrow(batch, rows, cap, heads, cosa::chunk_tokens(G));
}
int start32(int len, int w, int G, int j) { return of(len, w, G).start<int32_t>(j); }
int slots32(int len, int w, int G) { return of(len, w, G).slots<int32_t>(); }
int unit_keys() { return cosa::kUnitKeys; }
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("chunk")
    (d / "split.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-Wall", "-Werror",
                    f"-I{CSRC}", "-o", str(d / "split.so"), str(d / "split.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "split.so"))
    i, q = ctypes.c_int, ctypes.c_int64
    lib.narrow.argtypes = [q, q, q, q, i]
    for name, args, res in (("start", [i, i, i, i], q), ("slots", [i, i, i], q), ("find", [i, i, i, q], i),
                            ("range_length", [q, i, i], q), ("tile0", [q, q, i], i),
                            ("tile1", [q, q, i, i], i)):
        getattr(lib, name).argtypes, getattr(lib, name).restype = args, res
    return lib


def sequences():
    rng = random.Random(7)
    out = [(0, 0), (0, 1), (1, 1), (128, 128), (129, 3), (5, 900), (2 ** 31 - 1, 4000), (4000, 4000), (100, 101)]
    return out + [(rng.randrange(0, 3000), rng.randrange(0, 1500)) for _ in range(40)]


@pytest.mark.parametrize("G", [1, 2, 3, 4, 7, 20, 128, 255, 256, 257, 600])
def test_units_of_a_sequence(split, G):
    T, rows = split.tokens(G), split.chunk_rows()
    assert T >= 1 and T * split.heads(G) <= rows and split.heads(G) * split.parts(G) >= G
    assert (T + 1) * split.heads(G) > rows
    for length, w in sequences():
        n = split.units(length, w, G)
        assert n == -(-w // T)
        at = 0
        for j in range(n):
            keys = max(0, length - w + min((j + 1) * T, w))
            few = min(T, w - j * T) * split.heads(G) <= rows // 2
            assert not few or j == n - 1
            assert split.key_slots(length, w, G, j) == (2 if few else 3)
            assert split.keys(length, w, G, j) == keys
            assert split.tiles(length, w, G, j) == max(1, -(-keys // 128))
            assert split.start(length, w, G, j) == at, (length, w, G, j)
            cost = (keys + split.unit_keys()) * (2 if few else 3)
            for x in (at, at + cost // 2, at + cost - 1):
                assert split.find(length, w, G, x) == j
            # the unit's last tile starts inside its slots
            assert (split.tiles(length, w, G, j) - 1) * 128 < keys + split.unit_keys()
            at += cost
        assert split.slots(length, w, G) == at


@pytest.mark.parametrize("log2_most,shortest", [(0, 384), (8, 768), (8, 384), (4, 1000)])
def test_every_tile_has_one_range(split, log2_most, shortest):
    rng = random.Random(11)
    for _ in range(30):
        G = rng.choice([1, 4, 7, 20, 150, 300])
        seqs = [(rng.randrange(0, 4000), rng.randrange(0, 700)) for _ in range(rng.randrange(1, 9))]
        units, at = [], 0
        for length, w in seqs:
            for j in range(split.units(length, w, G)):
                slots = split.key_slots(length, w, G, j)
                units.append((at, split.tiles(length, w, G, j), slots))
                at += (split.keys(length, w, G, j) + split.unit_keys()) * slots
        length = split.range_length(at, log2_most, shortest)
        n = -(-at // length)
        assert n <= 1 << log2_most and length >= shortest >= 3 * 128
        owner = {}
        for b in range(n):
            lo, hi = b * length, min((b + 1) * length, at)
            started = unfinished = 0
            for u, (start, tiles, slots) in enumerate(units):
                end = units[u + 1][0] if u + 1 < len(units) else at
                if start >= hi or end <= lo:
                    continue
                t0, t1 = split.tile0(lo, start, slots), split.tile1(hi, start, slots, tiles)
                for t in range(t0, t1):
                    assert (u, t) not in owner
                    owner[u, t] = b
                if t0 < t1:
                    started += t0 > 0
                    unfinished += t0 == 0 and t1 < tiles
            # one place for a unit that began before, one for a unit that goes on
            assert started <= 1 and unfinished <= 1
        for u, (start, tiles, slots) in enumerate(units):
            owners = [owner[u, t] for t in range(tiles)]
            # the ranges of a unit follow each other, the last one is where its last tile starts
            assert sorted(set(owners)) == list(range(owners[0], owners[-1] + 1)) and owners == sorted(owners)
            assert owners[-1] == (start + (tiles - 1) * 128 * slots) // length


@pytest.mark.parametrize("G", [1, 4, 7, 150, 300])
def test_narrow_slots(split, G):
    rng = random.Random(13)
    narrow = wide = 0
    for _ in range(400):
        rows, cap = int(2 ** rng.uniform(0, 22)), int(2 ** rng.uniform(0, 31))
        heads, batch = rng.choice([1, 8, 64]), int(2 ** rng.uniform(0, 12))
        if not split.narrow(batch, rows, cap, heads, G):
            wide += 1
            continue
        narrow += 1
        for length, w in ((cap, rows), (0, rows), (cap, 1), (min(cap, rows // 2), rows), (rng.randrange(0, cap + 1), rng.randrange(1, rows + 1))):
            n = split.units(length, w, G)
            assert split.slots(length, w, G) * heads * batch < 2 ** 31
            assert split.slots32(length, w, G) == split.slots(length, w, G)
            for j in {0, n // 3, n - 1}:
                assert split.start32(length, w, G, j) == split.start(length, w, G, j)
    assert narrow > 20 and wide > 20
