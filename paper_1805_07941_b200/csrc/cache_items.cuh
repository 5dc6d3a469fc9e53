// Which head of a cache call a lane takes, in plain C++.  A warp's lanes stand in groups of G, one head each; the lanes behind
// the last whole group are idle, and take a number that is past every list: a call has at most 2^30 items, and a warp's first
// item of a round lies at most a few steps of the grid (148 * 8 blocks of up to 64 heads) behind the last, so that unsigned sums
// stay below 2^31 + 2^20.  (Signed, those of idle lanes would turn negative in lists of nearly 2^30 items.)
#pragma once
#include "any_side.cuh"

namespace qc {

constexpr unsigned int kCacheMaxItems = 1u << 30;

// Which of the warp's heads lane l (0 to 31) works on; kCacheMaxItems: none.
QC_ANY_SIDE unsigned int cache_mine(unsigned int l, unsigned int G) {
  const unsigned int mine = l / G;
  return mine < 32 / G ? mine : kCacheMaxItems;
}
// The `mine`-th item from `first` on, and whether a call of so many items has it.
QC_ANY_SIDE unsigned int cache_unit(int first, unsigned int mine) { return static_cast<unsigned int>(first) + mine; }
QC_ANY_SIDE bool cache_has(unsigned int u, int items) { return u < static_cast<unsigned int>(items); }

}  // namespace qc
