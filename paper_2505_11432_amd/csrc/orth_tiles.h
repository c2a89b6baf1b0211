// Which tiles the products of orthogonalised updates take (newton_schulz.hip), and what memory they need.  Host code without HIP.
#pragma once

#include <algorithm>

namespace moe {

constexpr int kOrthTile = 256, kOrthSmallTile = 64, kOrthStep = 64;      // sides of the tiles, and a step along the contraction
constexpr int kOrthPartFloats = kOrthTile * kOrthTile;
constexpr int kGroups = 256;                // workgroups on large tiles: a CU each
constexpr int kMostParts = 512;             // of a launch: 128 MB
constexpr int kMostSplit = 32;

// tiles of a matrix of M x N, or of the lower triangle of a symmetric one
struct OrthTiles { long large, small; };
inline OrthTiles orth_tiles(bool symmetric, int M, int N) {
  const long tm = (M + kOrthTile - 1) / kOrthTile, tn = (N + kOrthTile - 1) / kOrthTile, sm = M / kOrthSmallTile, sn = N / kOrthSmallTile;
  return symmetric ? OrthTiles{tm * (tm + 1) / 2, sm * (sm + 1) / 2} : OrthTiles{tm * tn, sm * sn};
}

// Which tiles are cut along K: those behind the last whole round of workgroups, where that is the faster way.  By measured times (us): a step 1.9, a tile's
// results 12, adding parts up a launch, and each of them 256 KB written and read.
struct Cut { int full, split; double time; };
inline double split_time(double rounds, int split, long parts, int steps) {
  return rounds + (double)((parts + kGroups - 1) / kGroups) * (1.9 * steps / split + 2) + 8 + 0.3 * split + 0.1 * (double)parts;
}
inline Cut cut_of(long tiles, int steps) {
  const int full = (int)(tiles / kGroups * kGroups), rem = (int)(tiles - full);
  const double rounds = (double)(full / kGroups) * (1.9 * steps + 12);
  Cut best{(int)tiles, 1, rounds + (rem ? 1.9 * steps + 12 : 0)};
  if (rem == 0) return best;
  for (int split = 2; split <= kMostSplit; ++split) {
    const long parts = (long)rem * split;
    if (steps / split < 2 || parts > kMostParts) break;
    const double time = split_time(rounds, split, parts, steps);
    if (time < best.time) best = {full, split, time};
  }
  return best;
}
// Small tiles: alone on its CU a workgroup takes 0.35 us a step, 512 of them together 0.65.  (us, all products on small tiles and on large ones: 512 x 512 87, 235;
// 1024 x 1024 122, 391, 8 of them 593, 799, 16 of them 1239, 697; 2048 x 2048 490, 757; 8 of 512 x 2048 321, 590; 512 x 16384 488, 516.)
inline double small_tiles_time(long tiles, int steps) { return std::max(0.35 * steps + 3, (double)tiles / (2 * kGroups) * (0.65 * steps + 4)) + 1.5; }

// Parts of cut tiles that a product of up to `count` matrices can ask for: none where small tiles are faster than any cut one, at most as many as there are
// tiles, each cut as often as it can be.  More matrices never need less.
inline long orth_most_parts(bool symmetric, int M, int N, int K, int count) {
  const OrthTiles t = orth_tiles(symmetric, M, N);
  const int steps = K / kOrthStep;
  int most = 0;
  double least = 0;
  for (int split = 2; split <= kMostSplit && steps / split >= 2; ++split) {
    const double time = split_time(0, split, split, steps);      // (a single tile)
    least = most ? std::min(least, time) : time;
    most = split;
  }
  if (most == 0 || small_tiles_time(t.small * count, steps) < least) return 0;
  return std::min<long>(kMostParts, std::min<long>(kGroups - 1, t.large * count) * most);
}

}  // namespace moe
