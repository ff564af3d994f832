// Work items of a grouped product: which expert's rows a block takes.
#pragma once

#include "moe_internal.h"

namespace moe {

// Rows [first, first + n) of an expert.
struct Rows {
  int first, n;
};

// A count as the sums below take it: none below zero, none above the call's
// rows, so that 512 of them fit 32 bits.
__device__ inline int count_of(const Grouped& g, int e) {
  return g.count ? max(0, min(g.count[e], g.n)) : g.n;
}

// Inclusive sum over the lanes up to this one (DPP row shifts, then the row
// ends broadcast to the rows above).
template <int CTRL, int ROWS>
__device__ inline int scan_step(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ inline int lanes_up_to(int v) {
  v = scan_step<0x111, 0xF>(v);  // row_shr:1
  v = scan_step<0x112, 0xF>(v);
  v = scan_step<0x114, 0xF>(v);
  v = scan_step<0x118, 0xF>(v);
  v = scan_step<0x142, 0xA>(v);  // row_bcast:15 into rows 1 and 3
  return scan_step<0x143, 0xC>(v);  // row_bcast:31 into rows 2 and 3
}

constexpr int kLaneExperts = kRouterMaxExperts / 64;  // most experts of a lane

// Rows of expert e (all lanes of the wave take part and get them).
__device__ inline Rows expert_rows(const Grouped& g, int e) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int i = lane; i < e; i += 64) before += count_of(g, i);
  before = min(__builtin_amdgcn_readlane(lanes_up_to(before), 63), g.n);
  return {before, __builtin_amdgcn_readfirstlane(min(count_of(g, e), g.n - before))};
}

// One row tile of an expert: rows [row, row + n) of the call.
struct RowTile {
  int expert, row, n;
  int part;            // column tile
};

// Row tiles of at most M rows come in two runs over the experts: first the
// full ones and the remainders of more than 3/4, which take the largest block,
// then the smaller remainders, so that these fill the last round.  An item is
// a row tile and one of `parts` column tiles; up to `super` row tiles of an
// expert alternate fastest, so that the blocks that run together on a die
// share the columns' operand and the rows'.
template <int M>
__device__ inline int big_tiles(int n) { return n / M + (n % M > 3 * M / 4); }

// The block's item of the numbering above.  The hardware hands block b to die
// b % 8: whole sets of 256 items (one per compute unit) go to the dies in runs
// of 32, what is left in eighths.  false: no work.  One wave computes it; every
// wave of a block gets the same.
__device__ inline int die_slots(int n) { return (n >> 8) * 32 + (((n & 255) + 7) >> 3); }
__device__ inline int die_item(int n, int die, int slot) {
  const int sets = n >> 8, left = n & 255, per = (left + 7) >> 3;
  if (slot < 32 * sets) return (slot >> 5) * 256 + die * 32 + (slot & 31);
  const int q = slot - 32 * sets, item = die * per + q;
  return q < per && item < left ? 256 * sets + item : -1;
}

template <int M>
__device__ inline bool take_row_tile(const Grouped& g, int parts, int super, RowTile& t) {
  const int lane = threadIdx.x & 63;
  // a lane holds `per` consecutive experts
  const int per = (g.E + 63) >> 6;
  int c[kLaneExperts], own = 0;
#pragma unroll
  for (int j = 0; j < kLaneExperts; ++j) {
    const int e = lane * per + j;
    c[j] = j < per && e < g.E ? count_of(g, e) : 0;
    own += c[j];
  }
  const int before = lanes_up_to(own) - own;
  int first = min(before, g.n), big = 0, rest = 0;
  const int first0 = first;
#pragma unroll
  for (int j = 0; j < kLaneExperts; ++j) {
    c[j] = min(c[j], g.n - first);
    first += c[j];
    const int b = big_tiles<M>(c[j]);
    big += b;
    rest += c[j] > b * M;
  }
  const int up_big = lanes_up_to(big), up_rest = lanes_up_to(rest);
  const int n_big = __builtin_amdgcn_readlane(up_big, 63) * parts;
  const int n_rest = __builtin_amdgcn_readlane(up_rest, 63) * parts;
  const int slot = blockIdx.x >> 3, die = blockIdx.x & 7, slots_big = die_slots(n_big);
  const bool small = slot >= slots_big;
  const int item = small ? die_item(n_rest, die, slot - slots_big) : die_item(n_big, die, slot);
  if (item < 0) return false;
  const int up = small ? up_rest : up_big, mine = small ? rest : big;
  const int at = __ffsll((unsigned long long)__ballot(up * parts > item)) - 1;
  // that lane's expert: the others compute something in range and are not read
  int in = item - (up - mine) * parts, row = first0, expert = lane * per, rows = 0, tiles = 1, found = 0;
#pragma unroll
  for (int j = 0; j < kLaneExperts; ++j) {
    const int b = big_tiles<M>(c[j]);
    const int k = small ? (c[j] > b * M) : b;
    const bool here = !found && in < k * parts;
    if (here) {
      expert = lane * per + j;
      rows = c[j];
      tiles = k;
      found = 1;
    }
    if (!found) {
      in -= k * parts;
      row += c[j];
    }
  }
  in = __builtin_amdgcn_readlane(in, at);
  row = __builtin_amdgcn_readlane(row, at);
  rows = __builtin_amdgcn_readlane(rows, at);
  tiles = __builtin_amdgcn_readlane(tiles, at);
  t.expert = __builtin_amdgcn_readlane(expert, at);
  const int sup = in / (super * parts), left = in - sup * (super * parts);
  const int width = min(super, tiles - sup * super);
  t.part = __builtin_amdgcn_readfirstlane(left / width);
  const int k = sup * super + left - t.part * width;
  const int r0 = small ? big_tiles<M>(rows) * M : k * M;
  t.row = __builtin_amdgcn_readfirstlane(row + r0);
  t.n = __builtin_amdgcn_readfirstlane(min(M, rows - r0));
  return true;
}

// Blocks for any counts: a tile of the first run has more than 3/4 M rows, and
// an expert at most one of the second.
inline unsigned row_tile_blocks(const Grouped& g, int M, int parts) {
  const int64_t tiles = g.n / (3 * M / 4 + 1) + (g.E < g.n ? g.E : g.n);
  return (unsigned)((tiles * parts + 7) / 8 + 2) * 8;
}

}  // namespace moe
