// What the expert products' kernels share: the rows of each expert, found on
// the device.
#pragma once

#include "tm_ops.h"

namespace tmk {
namespace expert {

// A run of rows [first, last) of one expert (experts: the rows of none).
struct Group {
  int e, first, last;
};

// First and last row of group e.  Whatever `ends` holds, the rows stay within the matrix.
__device__ inline Group group_of(const ExpertArgs& A, int e) {
  Group g;
  g.e = e;
  g.first = e == 0 ? 0 : min(max(A.ends[e - 1], 0), A.rows);
  g.last = e == A.experts ? A.rows : min(max(A.ends[e], g.first), A.rows);
  return g;
}

// Row tile `tile` (of T rows) of the launch: its group cut to the tile's rows.
// Every lane of a wave calls it; the lanes look at 64 groups at a time.  False
// past the last tile.
template <int T>
__device__ inline bool find_tile(const ExpertArgs& A, int tile, Group& out) {
  const int lane = threadIdx.x & 63;
  int before = 0;   // tiles of the groups looked at so far
  for (int base = 0; base <= A.experts; base += 64) {
    const int e = base + lane;
    Group g{e, 0, 0};
    if (e <= A.experts) g = group_of(A, e);
    const int tiles = (g.last - g.first + T - 1) / T;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int up = __shfl_up(sum, o);
      if (lane >= o) sum += up;
    }
    const uint64_t past = __ballot(before + sum > tile);
    if (past != 0) {
      const int src = __ffsll((unsigned long long)past) - 1;
      const int first = __shfl(g.first, src) + (tile - before - __shfl(sum - tiles, src)) * T;
      out = Group{base + src, first, min(first + T, __shfl(g.last, src))};
      return true;
    }
    before += __shfl(sum, 63);
  }
  return false;
}

}  // namespace expert
}  // namespace tmk
