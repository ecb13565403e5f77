// A workgroup's place in a step whose sequences bring different numbers of tiles (device
// code).
#pragma once

#include "../launch_tokens.h"

namespace uf {
namespace tok {

// Tile k of a step, tiles being counted sequence by sequence: units(entry) of them in a
// sequence.  64 sequences at a time, by every wave for itself; entry -1: there are fewer.
struct Place {
  int entry, tile;
};
template <class F>
__device__ inline Place place_of(const int32_t* step, int n, int k, F units) {
  const int lane = threadIdx.x & 63;
  n = min(n, __builtin_amdgcn_readfirstlane(step[0]));
  for (int e0 = 0; e0 < n; e0 += 64) {
    const int w = e0 + lane < n ? units(step + kHeader + kEntry * (e0 + lane)) : 0;
    int s = w;                                         // of the lanes up to this one
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int t = __shfl_up(s, d);
      if (lane >= d) s += t;
    }
    const uint64_t past = __ballot(s > k);
    if (past != 0) {
      const int at = __ffsll(static_cast<unsigned long long>(past)) - 1;
      return Place{e0 + at, k - __builtin_amdgcn_readlane(s - w, at)};
    }
    k -= __builtin_amdgcn_readlane(s, 63);
  }
  return Place{-1, 0};
}

}  // namespace tok
}  // namespace uf
