// How the work of an attention call over chunks of new tokens is dealt out: plain arithmetic, the same on the host
// and in the kernels.
//
// A unit is (sequence, KV head, up to 256 query heads of its group, T tokens): its rows are the T tokens' heads, T as
// many whole tokens as 256 rows hold. It walks the keys up to its last token in tiles of 128. Units lie one
// behind the other on a line of slots, each as long as it takes in time; the line is cut into equal ranges, and a range has
// the tiles whose first slot it holds. So every tile has one owner whatever the lengths are, and a unit's place on the
// line has a closed form: only the last unit of a sequence has fewer than T tokens.
#pragma once

#include <stdint.h>

namespace cosa {

constexpr int kChunkRows = 256;  // rows of a unit
constexpr int kChunkTile = 128;  // keys of a tile
// Slots of a key in a unit, and in one whose rows leave half of the workgroup idle (its tiles take some 5,000 cycles, others
// 7,000). Counted alike, the ranges of one-token units end early: 48 sequences of which 43 add one token 777 us instead of
// 769 with 32 / 8 heads, 813 instead of 786 with 40 / 8. Prompts, whose last units alone differ, do not change.
constexpr int kFullSlots = 3, kFewSlots = 2;
// What taking up a unit costs beside its keys, in keys; at least a tile, so that a unit's last tile starts inside its
// slots. 19 prompts of up to 4K tokens with 288 / 352 / 400 / 448 / 512 keys: 741 / 719 / 706 / 707 / 715 us with 28 / 4 heads and
// pages of 16, 826 / 802 / 796 / 797 / 803 with 32 / 8 and 128, 447 / 441 / 440 / 440 / 444 with 16 / 16 and 64; a prompt of 8K 545 / 522 /
// 522 / 523 / 527: flat from 352 on.
constexpr int kUnitKeys = 400;

// Heads of a unit, units that share a group, and tokens of a unit, for G query heads per KV head.
constexpr int chunk_heads(int G) { return G < kChunkRows ? G : kChunkRows; }
constexpr int chunk_parts(int G) { return (G + kChunkRows - 1) / kChunkRows; }
constexpr int chunk_tokens(int G) { return kChunkRows / chunk_heads(G); }

// One sequence's units for one KV head and part: `len` tokens, the last `w` of them new (w > len: the first w - len
// stand in front of token 0 and see nothing), T new tokens of `heads` rows a unit. I: int64_t, or int32_t where chunk_narrow().
struct ChunkSeq {
  int len, w, T, heads;

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
  constexpr int key_slots(int j) const {
    const int64_t left = (int64_t)w - (int64_t)j * T;
    return (left < T ? left : T) * heads <= kChunkRows / 2 ? kFewSlots : kFullSlots;
  }
  template <class I>
  constexpr I cost(int j) const {
    return ((I)keys(j) + kUnitKeys) * key_slots(j);
  }
  // Slots in front of unit j (all units in front of it have T tokens, more than half of the rows).
  template <class I>
  constexpr I start(int j) const {
    const int ahead = w - len, z = ahead > 0 ? (int)((uint32_t)ahead / (uint32_t)T) : 0;  // units that end in front of token 0
    I s = (I)kUnitKeys * j;
    if (j > z) s += (I)(j - z) * (len - w) + (I)T * ((I)j * (j + 1) - (I)z * (z + 1)) / 2;
    return s * kFullSlots;
  }
  template <class I>
  constexpr I slots() const {  // of all units
    const int n = units();
    return n == 0 ? 0 : start<I>(n - 1) + cost<I>(n - 1);
  }
};

// Whether 31 bits hold every sum of slots of a call, and of their terms: `batch` sequences of up to n_rows rows (they may
// overlap) and `cap` tokens, units for `heads` KV heads and parts.
constexpr bool chunk_narrow(int64_t batch, int64_t n_rows, int64_t cap, int64_t heads, int T) {
  const int64_t units = n_rows / T + 1, most = (cap > n_rows ? cap : n_rows) + kUnitKeys;  // of a sequence; keys of a unit
  const double limit = 2147483648.0;
  return (double)units * (double)(n_rows + 2 * T) < limit &&
         (double)units * (double)most * kFullSlots * (double)heads * (double)batch < limit / 2;
}

// Whether 62 bits hold them, whatever the offsets say. Calls of which they do not are refused.
constexpr bool chunk_fits(int64_t batch, int64_t n_rows, int64_t cap, int64_t heads, int T) {
  return (double)(n_rows / T + 1) * (double)(cap + kUnitKeys) * kFullSlots * (double)heads * (double)batch < 4611686018427387904.0;
}

// The ranges of a line of `total` slots: 2^log2_most of `length` slots each; the last ones may have fewer, or none.
template <class I>
constexpr I chunk_range(I total, int log2_most, int shortest) {
  const I length = (total + ((I)1 << log2_most) - 1) >> log2_most;
  return length < shortest ? shortest : length;
}

// The largest i in [0, n) with start(i) <= x, for start(0) <= x and a start that does not fall, is searched for in rounds
// of 64 places, a lane each: the first round looks at every search_step(n)-th place, the next ones at a 64th of that.
constexpr int search_step(int n) {
  int step = 1;
  while ((int64_t)step * 64 < n) step *= 64;
  return step;
}

// Tiles [t0, t1) that the range [a, b) has of a unit of `tiles` tiles whose slots start at u, key_slots a key.
template <class I>
constexpr I chunk_tiles_ahead(I slots, int key_slots) {
  return key_slots == kFewSlots ? (slots + kChunkTile * kFewSlots - 1) / (kChunkTile * kFewSlots)
                                : (slots + kChunkTile * kFullSlots - 1) / (kChunkTile * kFullSlots);
}
template <class I>
constexpr int chunk_tile0(I a, I u, int key_slots) {
  return a > u ? (int)chunk_tiles_ahead<I>(a - u, key_slots) : 0;
}
template <class I>
constexpr int chunk_tile1(I b, I u, int key_slots, int tiles) {
  const I t = chunk_tiles_ahead<I>(b - u, key_slots);
  return t < tiles ? (int)t : tiles;
}

}  // namespace cosa
