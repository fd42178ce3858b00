// How the work of an attention call of one token is dealt out: plain arithmetic, the same on the host and in the
// kernels.
#pragma once

namespace cosa {

constexpr int kJoinGroups = 16;  // groups of 32 lanes in a workgroup of the join

// Query heads of unit qg of a group of G, `rows` heads a unit (the last one may have fewer).
constexpr int unit_heads(int G, int rows, int qg) {
  return G - qg * rows < rows ? G - qg * rows : rows;
}

// The join of `units` units: every unit's heads in `groups` workgroups of `heads` each (the last one may have
// fewer), and 2^log2_per_head groups of lanes a head. Few units leave many partial results each: then every
// head has workgroups of its own.
struct JoinShape {
  int heads, groups, log2_per_head;
};
constexpr JoinShape join_shape(long long units, int G, int rows) {
  const int most = G < rows ? G : rows;
  const long long spare = 256 / units;
  const int parts = spare < 1 ? 1 : spare < most ? (int)spare : most;
  int heads = (most + parts - 1) / parts;
  if (heads > kJoinGroups) heads = kJoinGroups;
  int log2_per_head = 4;
  while (heads << log2_per_head > kJoinGroups) --log2_per_head;
  return {heads, (most + heads - 1) / heads, log2_per_head};
}

// The head of a unit of `in_unit` heads that lane group `group` of its workgroup y joins; -1: none.
constexpr int join_head(int heads, int log2_per_head, int in_unit, int y, int group) {
  const int slot = group >> log2_per_head, head = y * heads + slot;
  return slot < heads && head < in_unit ? head : -1;
}

}  // namespace cosa
