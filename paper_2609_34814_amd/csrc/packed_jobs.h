// Into how many jobs the tiles of the gradient over packed sequences are cut (packed_bwd.hip): whole numbers, the same on the host.
#pragma once

#include <stdint.h>

namespace wa {

constexpr uint32_t kSlots = 512, kMostParts = 2 * kSlots;

// Tiles longer than this are cut: `sum` lengths of all tiles, of which a pair of a key and a query takes `share` of seven products, are
// shared by 512 workgroups. No tile is longer than `longest`, so a larger share cuts nothing either, and does not have to fit 32 bits
// (2^26 - 1 tokens of one sequence, 2 heads, without a causal mask: 2.5e9).
__host__ __device__ inline int longest_whole(int64_t sum, int share, int longest) {
  const int64_t most = (7 * sum + share * (int64_t)kSlots - 1) / (share * (int64_t)kSlots);
  return (int)(most < longest ? most : longest);
}
__host__ __device__ inline int parts_of(int length, int most) { return (length + most - 1) / most; }
// jobs of the first x lengths, 1 to x, of a causal sequence
__host__ __device__ inline int jobs_upto(int x, int most) {
  const int q = x / most, r = x - q * most;
  return q * (q + 1) / 2 * most + r * (q + 1);
}

}  // namespace wa
