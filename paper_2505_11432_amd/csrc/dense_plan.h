// Which tiles of a dense product are cut along the contraction, as the product's kernel and those that add up the parts work it out on the device.
#pragma once
#include <hip/hip_runtime.h>

#include "row_plan.h"

namespace moe {

constexpr int kDenseGroupN = 8;         // n-tiles per group of the tile list

struct DensePlan {
  int full_tiles, split, items;         // tiles [0, full_tiles) are whole, each of the others `split` neighbouring items
};

// A lane per number of parts; every wave comes to the same result.
__device__ __forceinline__ DensePlan dense_plan(int tiles, int groups, int steps, CutCost cost, bool cut) {
  DensePlan p{tiles, 1, tiles};
  const int rem = tiles % groups;
  if (!cut || rem == 0) return p;
  unsigned long long best = (unsigned long long)cut_ns((int)(threadIdx.x & 63) + 1, rem, groups, steps, cost);
  int parts = (int)(threadIdx.x & 63) + 1;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const unsigned long long other = __shfl_xor(best, off);
    const int other_parts = __shfl_xor(parts, off);
    if (other < best || (other == best && other_parts < parts)) {
      best = other;
      parts = other_parts;
    }
  }
  p.split = __builtin_amdgcn_readfirstlane(parts);
  if (p.split > 1) {
    p.full_tiles = tiles - rem;
    p.items = p.full_tiles + rem * p.split;
  }
  return p;
}

// place of tile (mt, nt) in the list of tiles_m x tiles_n tiles: groups of kDenseGroupN columns, row by row
__device__ __forceinline__ int dense_tile_index(int mt, int nt, int tiles_m, int tiles_n) {
  const int ng = nt / kDenseGroupN, gw = min(kDenseGroupN, tiles_n - ng * kDenseGroupN);
  return ng * tiles_m * kDenseGroupN + mt * gw + (nt - ng * kDenseGroupN);
}

}  // namespace moe
