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
int units(int len, int w, int T) { return ChunkSeq{len, w, T}.units(); }
int keys(int len, int w, int T, int j) { return ChunkSeq{len, w, T}.keys(j); }
int tiles(int len, int w, int T, int j) { return ChunkSeq{len, w, T}.tiles(j); }
int64_t start(int len, int w, int T, int j) { return ChunkSeq{len, w, T}.start(j); }
int64_t slots(int len, int w, int T) { return ChunkSeq{len, w, T}.slots(); }
// the unit that holds slot x, in rounds as the kernel's lanes search for it
int find(int len, int w, int T, int64_t x) {
  const ChunkSeq s{len, w, T};
  const int n = s.units();
  int first = 0;
  for (int step = cosa::search_step(n); step; step /= 64) {
    int hits = 0;
    for (int lane = 0; lane < 64; ++lane) {
      const int64_t i = (int64_t)first + (int64_t)lane * step;
      hits += i < n && s.start((int)i) <= x;
    }
    first += (hits - 1) * step;
  }
  return first;
}
int64_t range_length(int64_t total, int log2_most, int shortest) { return cosa::chunk_range(total, log2_most, shortest); }
int tile0(int64_t a, int64_t u) { return cosa::chunk_tile0(a, u); }
int tile1(int64_t b, int64_t u, int tiles) { return cosa::chunk_tile1(b, u, tiles); }
int unit_slots() { return cosa::kUnitSlots; }
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
    for name, args, res in (("start", [i, i, i, i], q), ("slots", [i, i, i], q), ("find", [i, i, i, q], i),
                            ("range_length", [q, i, i], q), ("tile0", [q, q], i),
                            ("tile1", [q, q, i], i)):
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
        n = split.units(length, w, T)
        assert n == -(-w // T)
        at = 0
        for j in range(n):
            keys = max(0, length - w + min((j + 1) * T, w))
            assert split.keys(length, w, T, j) == keys
            assert split.tiles(length, w, T, j) == max(1, -(-keys // 128))
            assert split.start(length, w, T, j) == at, (length, w, T, j)
            for x in (at, at + keys, at + keys + split.unit_slots() - 1):
                assert split.find(length, w, T, x) == j
            # the unit's last tile starts inside its slots
            assert (split.tiles(length, w, T, j) - 1) * 128 < keys + split.unit_slots()
            at += keys + split.unit_slots()
        assert split.slots(length, w, T) == at


@pytest.mark.parametrize("log2_most,shortest", [(0, 128), (8, 256), (8, 128), (4, 512)])
def test_every_tile_has_one_range(split, log2_most, shortest):
    rng = random.Random(11)
    for _ in range(30):
        T = rng.choice([1, 12, 36, 64, 256])
        seqs = [(rng.randrange(0, 4000), rng.randrange(0, 700)) for _ in range(rng.randrange(1, 9))]
        units, at = [], 0
        for length, w in seqs:
            for j in range(split.units(length, w, T)):
                units.append((at, split.tiles(length, w, T, j)))
                at += split.keys(length, w, T, j) + split.unit_slots()
        length = split.range_length(at, log2_most, shortest)
        n = -(-at // length)
        assert n <= 1 << log2_most and length >= shortest >= 128
        owner = {}
        for b in range(n):
            lo, hi = b * length, min((b + 1) * length, at)
            started = unfinished = 0
            for u, (start, tiles) in enumerate(units):
                end = units[u + 1][0] if u + 1 < len(units) else at
                if start >= hi or end <= lo:
                    continue
                t0, t1 = split.tile0(lo, start), split.tile1(hi, start, tiles)
                for t in range(t0, t1):
                    assert (u, t) not in owner
                    owner[u, t] = b
                if t0 < t1:
                    started += t0 > 0
                    unfinished += t0 == 0 and t1 < tiles
            # one place for a unit that began before, one for a unit that goes on
            assert started <= 1 and unfinished <= 1
        for u, (start, tiles) in enumerate(units):
            owners = [owner[u, t] for t in range(tiles)]
            # the ranges of a unit follow each other, the last one is where its last tile starts
            assert sorted(set(owners)) == list(range(owners[0], owners[-1] + 1)) and owners == sorted(owners)
            assert owners[-1] == (start + (tiles - 1) * 128) // length
