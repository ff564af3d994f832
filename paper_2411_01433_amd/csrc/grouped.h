// Work items of a grouped product: which expert's rows a block takes.
#pragma once

#include "tile.h"

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

// The counts of all experts in a wave's registers: a lane holds `per`
// consecutive ones, cut at the call's rows, and the first row of its first.
struct Counts {
  int per, n[kLaneExperts], first;

  __device__ inline void init(const Grouped& g) {
    const int lane = threadIdx.x & 63;
    per = (g.E + 63) >> 6;
    int own = 0;
#pragma unroll
    for (int j = 0; j < kLaneExperts; ++j) {
      const int e = lane * per + j;
      n[j] = j < per && e < g.E ? count_of(g, e) : 0;
      own += n[j];
    }
    first = min(lanes_up_to(own) - own, g.n);
    int at = first;
#pragma unroll
    for (int j = 0; j < kLaneExperts; ++j) {
      n[j] = min(n[j], g.n - at);
      at += n[j];
    }
  }
  // Rows of expert e (uniform).
  __device__ inline Rows rows(int e) const {
    const int lane = e / per, k = e - lane * per;
    int at = first, own = n[0];
#pragma unroll
    for (int j = 1; j < kLaneExperts; ++j) {
      if (j <= k) {
        at += n[j - 1];
        own = n[j];
      }
    }
    return {__builtin_amdgcn_readlane(at, lane), __builtin_amdgcn_readlane(own, lane)};
  }
};

// One row tile of an expert: rows [row, row + n) of the call.
struct RowTile {
  int expert, row, n;
  int part;            // column tile
};

// The numbers of n items that a die takes, and the item at one of its places
// (-1: none).  The hardware hands block b to die b % 8; whole sets of 256
// items (one per compute unit) go to the dies in runs of 32, what is left in
// eighths, so that every die gets the same mix.
__device__ inline int die_slots(int n) { return (n >> 8) * 32 + (((n & 255) + 7) >> 3); }
__device__ inline int die_item(int n, int die, int slot) {
  const int sets = n >> 8, left = n & 255, per = (left + 7) >> 3;
  if (slot < 32 * sets) return (slot >> 5) * 256 + die * 32 + (slot & 31);
  const int q = slot - 32 * sets, item = die * per + q;
  return q < per && item < left ? 256 * sets + item : -1;
}

// The row tiles of a call, at most M rows each.  They come in two runs over the
// experts: first the full ones and the remainders of more than 3/4, which take
// the largest block, then the smaller remainders, so that these fill the last
// round.  An item is a row tile and one of `parts` column tiles; up to kSuper
// row tiles of an expert alternate fastest, so that the blocks that run
// together on a die share the columns' operand and the rows'.
template <int M>
struct RowTiles {
  static constexpr int kSuper = 8;
  int parts, n_big, n_rest, slots_big, slots;
  Counts counts;
  int big, rest, up_big, up_rest;  // of the lane's experts, and up to them

  static __device__ inline int big_of(int n) { return n / M + (n % M > 3 * M / 4); }
  static __device__ inline int rest_of(int n) { return n > big_of(n) * M; }

  // (all lanes of a wave, as get)
  __device__ inline void init(const Grouped& g, int parts_) {
    parts = parts_;
    counts.init(g);
    big = rest = 0;
#pragma unroll
    for (int j = 0; j < kLaneExperts; ++j) {
      big += big_of(counts.n[j]);
      rest += rest_of(counts.n[j]);
    }
    up_big = lanes_up_to(big);
    up_rest = lanes_up_to(rest);
    n_big = __builtin_amdgcn_readlane(up_big, 63) * parts;
    n_rest = __builtin_amdgcn_readlane(up_rest, 63) * parts;
    slots_big = die_slots(n_big);
    slots = slots_big + die_slots(n_rest);
  }

  // The item of a die's place; false: none there.
  __device__ inline bool get(int die, int slot, RowTile& t) const {
    const int lane = threadIdx.x & 63;
    const bool small = slot >= slots_big;
    const int item = small ? die_item(n_rest, die, slot - slots_big) : die_item(n_big, die, slot);
    if (item < 0) return false;
    const int up = small ? up_rest : up_big, mine = small ? rest : big;
    const int at = __ffsll((unsigned long long)__ballot(up * parts > item)) - 1;
    // that lane's expert: what the others compute is not read
    int in = item - (up - mine) * parts, row = counts.first, expert = lane * counts.per, rows = 0, tiles = 1;
    bool found = false;
#pragma unroll
    for (int j = 0; j < kLaneExperts; ++j) {
      const int k = (small ? rest_of(counts.n[j]) : big_of(counts.n[j])) * parts;
      const bool here = !found && in < k;
      if (here) {
        expert = lane * counts.per + j;
        rows = counts.n[j];
        tiles = k;
      }
      found = found || here;
      if (!found) {
        in -= k;
        row += counts.n[j];
      }
    }
    in = __builtin_amdgcn_readlane(in, at);
    row = __builtin_amdgcn_readlane(row, at);
    rows = __builtin_amdgcn_readlane(rows, at);
    tiles = __builtin_amdgcn_readlane(tiles, at) / parts;
    t.expert = __builtin_amdgcn_readlane(expert, at);
    const int sup = in / (kSuper * parts), left = in - sup * (kSuper * parts);
    const int width = min(kSuper, tiles - sup * kSuper);
    t.part = __builtin_amdgcn_readfirstlane(left / width);
    const int k = sup * kSuper + left - t.part * width;
    const int r0 = small ? big_of(rows) * M : k * M;
    t.row = __builtin_amdgcn_readfirstlane(row + r0);
    t.n = __builtin_amdgcn_readfirstlane(min(M, rows - r0));
    return true;
  }
};

// Blocks of one item each that any counts can fill: a tile of the first run has
// more than 3/4 M rows, and an expert at most one of the second.
inline unsigned row_tile_blocks(const Grouped& g, int M, int parts) {
  const int64_t tiles = g.n / (3 * M / 4 + 1) + (g.E < g.n ? g.E : g.n);
  return (unsigned)((tiles * parts + 7) / 8 + 2) * 8;
}

template <int TYPE> struct Elem { typedef f16 T; };
template <> struct Elem<tile::BF16> { typedef bf16 T; };

// Blocks of 64 TA columns and up to 64 TA rows (TA 1: 128), with the LDS of one
// (TA 4) or two blocks per unit, and as many blocks as the chip holds: each takes
// one item after another.
template <int TA> constexpr int kLds = TA == 4 ? 160 * 1024 : 80 * 1024;
template <int TA> constexpr int kRows = TA == 1 ? 128 : 64 * TA;
template <int TA> constexpr int kBlocks = TA == 4 ? 256 : 512;

// A block's items: place after place of its die's.  A job of TB takes the tiles
// whose rows fill TB of its 64s, and leaves off at the first other one.
template <int TA>
struct Items {
  RowTiles<kRows<TA>> tiles;
  int slot;
  RowTile t;           // the first one not taken; n = 0: none

  __device__ inline void init(const Grouped& g, int parts) {
    tiles.init(g, parts);
    tile::set_aside(tiles.parts);
    tile::set_aside(tiles.n_big);
    tile::set_aside(tiles.n_rest);
    tile::set_aside(tiles.slots_big);
    tile::set_aside(tiles.slots);
    tile::set_aside(tiles.counts.per);
    slot = (int)(blockIdx.x >> 3) - kBlocks<TA> / 8;
    tile::set_aside(slot);
    step();
  }
  __device__ inline void step() {
    RowTiles<kRows<TA>> now = tiles;  // (in scalar registers for as long as this takes)
    now.parts = __builtin_amdgcn_readfirstlane(tiles.parts);
    now.n_big = __builtin_amdgcn_readfirstlane(tiles.n_big);
    now.n_rest = __builtin_amdgcn_readfirstlane(tiles.n_rest);
    now.slots_big = __builtin_amdgcn_readfirstlane(tiles.slots_big);
    now.slots = __builtin_amdgcn_readfirstlane(tiles.slots);
    now.counts.per = __builtin_amdgcn_readfirstlane(tiles.counts.per);
    int at = __builtin_amdgcn_readfirstlane(slot);
    RowTile x = {0, 0, 0, 0};
    bool any = false;
    while (!any && (at += kBlocks<TA> / 8) < now.slots) any = now.get(blockIdx.x & 7, at, x);
    if (!any) x.n = 0;
    t = x;
    slot = at;
    tile::set_aside(slot);
    tile::set_aside(t.expert);
    tile::set_aside(t.row);
    tile::set_aside(t.n);
    tile::set_aside(t.part);
  }
  __device__ inline int rows() const { return __builtin_amdgcn_readfirstlane(t.n); }
  __device__ inline int size() const { return (rows() + 63) >> 6; }
  __device__ inline bool next(int tb, RowTile& x) {
    if (size() != tb) return false;
    x = {__builtin_amdgcn_readfirstlane(t.expert), __builtin_amdgcn_readfirstlane(t.row), rows(),
         __builtin_amdgcn_readfirstlane(t.part)};
    step();
    return true;
  }
};

// Whether a call has so few tiles that blocks of 64 columns and up to 128 rows
// do not outnumber the units.  Us with these / with blocks of 128 columns, fp16:
// 64 rows of one expert, 4096 x 4096 (64 tiles of 64 columns) 23.6 / 35.2, 14336
// x 4096 (224) 27.6 / 38.2, 28672 x 4096 (448) 52 / 48; 512 rows, 4096 x 4096
// (256) 30 / 39, 1024 rows (512) 55 / 42; 8 experts of 2048 x 4096, 25 rows each
// (256) 30 / 38.  MXFP4 beside 16 bits, 64 rows, 4096 x 4096: 27.6 / 34.5, on
// both sides 21.2 / 23.6 (512 rows 25.7 / 23.0: there the narrow ones lose, as the
// kind of operands is not asked for).
inline bool narrow_blocks(const Grouped& g, int cols) {
  const int active = g.E < g.n ? g.E : g.n;
  const int tiles = g.n / 128 + active / 2;
  return (int64_t)(tiles > active ? tiles : active) * (cols / 64) <= 256;
}

// Whether blocks of 256 columns and rows fill the chip, and the experts' rows
// fill enough of them (`rows` each on average).  Us with large / small blocks, 16
// experts of 6400 x 4096: forward at 32 rows each 178 / 166, 64 183 / 180, 128
// 202 / 224; d_x at 8 rows 126 / 136, 64 129 / 140, 256 209 / 270; MXFP4 on both sides at 16
// rows 61 / 68, 128 84 / 98; MXFP4 beside 16 bits, whose blocks of few rows wait
// for instructions more than for memory, at 64 rows 134 / 109, 256 278 / 264, 512
// 413 / 474.
inline bool large_blocks(const Grouped& g, int cols, int rows) {
  const int active = g.E < g.n ? g.E : g.n;
  const int tiles = g.n / 256 + active / 2;
  return (int64_t)(tiles > active ? tiles : active) * ((cols + 255) / 256) >= 256 &&
         g.n >= (int64_t)rows * active;
}

}  // namespace moe
