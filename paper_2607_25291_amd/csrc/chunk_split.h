// How the work of an attention call over chunks of new tokens is dealt out: plain arithmetic, the same on the host
// and in the kernels.
//
// A unit is (sequence, KV head, up to 256 query heads of its group, T tokens): its rows are the T tokens' heads, T as
// many whole tokens as 256 rows hold. It walks the keys up to its last token in tiles of 128. Units lie one
// behind the other on a line of slots, a slot a key and kUnitSlots more for a unit; the line is cut into equal
// ranges, and a range has the tiles whose first slot it holds. So every tile has one owner whatever the lengths are, and
// a unit's place on the line has a closed form.
#pragma once

#include <stdint.h>

namespace cosa {

constexpr int kChunkRows = 256;  // rows of a unit
constexpr int kChunkTile = 128;  // keys of a tile
// What taking up a unit costs beside its keys. At least a tile, so that a unit's last tile starts inside its slots.
constexpr int kUnitSlots = 448;

// Heads of a unit, units that share a group, and tokens of a unit, for G query heads per KV head.
constexpr int chunk_heads(int G) { return G < kChunkRows ? G : kChunkRows; }
constexpr int chunk_parts(int G) { return (G + kChunkRows - 1) / kChunkRows; }
constexpr int chunk_tokens(int G) { return kChunkRows / chunk_heads(G); }

// One sequence's units for one KV head and part: `len` tokens, the last `w` of them new (w > len: the first w - len
// stand in front of token 0 and see nothing), T new tokens a unit.
struct ChunkSeq {
  int len, w, T;

  constexpr int units() const { return (int)(((uint32_t)w + (uint32_t)T - 1u) / (uint32_t)T); }
  // Keys up to the last token of unit j.
  constexpr int keys(int j) const {
    const int64_t end = ((int64_t)j + 1) * T, k = (int64_t)len - w + (end < w ? end : w);
    return k > 0 ? (int)k : 0;
  }
  constexpr int tiles(int j) const {  // a unit without keys has one all the same, that writes its rows
    const int t = (int)(((int64_t)keys(j) + kChunkTile - 1) / kChunkTile);
    return t > 0 ? t : 1;
  }
  // Slots in front of unit j (all units in front of it have T tokens).
  constexpr int64_t start(int j) const {
    const int64_t ahead = (int64_t)w - len, z = ahead > 0 ? (uint32_t)ahead / (uint32_t)T : 0;  // units that end in front of token 0
    int64_t s = (int64_t)kUnitSlots * j;
    if (j > z) s += (j - z) * ((int64_t)len - w) + (int64_t)T * ((int64_t)j * (j + 1) - z * (z + 1)) / 2;
    return s;
  }
  constexpr int64_t slots() const {  // of all units
    const int n = units();
    return n == 0 ? 0 : start(n - 1) + keys(n - 1) + kUnitSlots;
  }
};

// The ranges of a line of `total` slots: 2^log2_most of `length` slots each; the last ones may have fewer, or none.
constexpr int64_t chunk_range(int64_t total, int log2_most, int shortest) {
  const int64_t length = (total + (1ll << log2_most) - 1) >> log2_most;
  return length < shortest ? shortest : length;
}

// The largest i in [0, n) with start(i) <= x, for start(0) <= x and a start that does not fall, is searched for in rounds
// of 64 places, a lane each: the first round looks at every search_step(n)-th place, the next ones at a 64th of that.
constexpr int search_step(int n) {
  int step = 1;
  while ((int64_t)step * 64 < n) step *= 64;
  return step;
}

// Tiles [t0, t1) that the range [a, b) has of a unit of `tiles` tiles whose slots start at u.
constexpr int chunk_tile0(int64_t a, int64_t u) { return a > u ? (int)((a - u + kChunkTile - 1) / kChunkTile) : 0; }
constexpr int chunk_tile1(int64_t b, int64_t u, int tiles) {
  const int64_t t = (b - u + kChunkTile - 1) / kChunkTile;
  return t < tiles ? (int)t : tiles;
}

}  // namespace cosa
