// What the attention of prefixes (prefix_attention.hip) leaves for the attention of the requests' own keys (attention.hpp), which joins it.
//
// The prefix of a group, once for each of its key heads and each `columns` of the query heads that read it, is a row of units of keys; the
// rows of all groups are one long row, of which every workgroup takes an equal share.  A workgroup's part of a row is a piece: workgroup w's of
// row r (counted over all groups) is piece w + r, since a next piece begins where a share or a row does.  Every workgroup finds the groups' units by
// itself, from as many as 1024 lengths, and all write the plan together: a workgroup more for it costs 2 us.
#pragma once

#include "operators.hpp"

namespace fc {

constexpr int kPrefixGroups = 1024;        // of a call, whose starts a workgroup keeps in LDS

// floats of a piece: the weighted sums of its columns, then (m, l) of each
__device__ __host__ __forceinline__ size_t prefix_piece_floats(unsigned columns, unsigned dim) { return (size_t)columns * (dim + 2); }

// Of a request: its group's first unit, the units of one of its rows (0: it has no prefix), its place in the group, how many times `columns`
// query heads the group's requests have for a key head, and the group's first row.
struct PrefixOf {
  unsigned start, units, index, blocks, row;
};

// words [0]: units of a share, [8 + 8 b ..]: PrefixOf of request b
struct PrefixPlan {
  const unsigned *words;
  __device__ __forceinline__ explicit PrefixPlan(const unsigned *p) : words(p) {}
  static __host__ size_t bytes(unsigned requests) { return (8 + 8 * (size_t)requests) * sizeof(unsigned); }
  __device__ __forceinline__ unsigned share() const { return words[0]; }
  __device__ __forceinline__ PrefixOf of(unsigned b) const {
    const unsigned *w = words + 8 + 8 * (size_t)b;
    const Vec<unsigned, 4> first = load_vec<unsigned, 4>(w);
    return {first[0], first[1], first[2], first[3], w[4]};
  }
};

}  // namespace fc
