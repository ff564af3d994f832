// Where the rows of an expert lie in a grouped product.
#pragma once

#include "moe_internal.h"

namespace moe {

// Rows [first, first + n) of an expert.
struct Rows {
  int first, n;
};

// A count as the sums below take it: none below zero, none above the call's
// rows, so that 512 of them fit 32 bits.
__device__ inline int rows_of(const Grouped& g, int e) {
  return g.count ? max(0, min(g.count[e], g.n)) : g.n;
}

// Rows of expert e, the sum of the counts before it; one wave (all lanes).
__device__ inline Rows expert_rows(const Grouped& g, int e) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int i = lane; i < e; i += 64) before += rows_of(g, i);
  for (int m = 1; m < 64; m <<= 1) before += __shfl_xor(before, m);
  before = min(before, g.n);
  return {before, min(rows_of(g, e), g.n - before)};
}

}  // namespace moe
