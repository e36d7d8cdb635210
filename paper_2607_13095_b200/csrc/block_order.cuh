// The order in which the tile kernels' blocks take the requests of a batch.
#pragma once

#include "hswa_internal.cuh"

namespace hswa_dev {

// Longest REQUEST first: the tiles of a request stay together (their blocks walk the same K/V pages at the same
// time, which keeps them in L2 and measured 4 % faster on the chunked-prefill workload than any order that
// interleaves requests), requests are taken in descending order of their longest tile's work, ceil(ctx_r / 128) +
// tiles_r (ties: ascending request), and inside a request the longest tile goes first, so that the launch ends on the
// shortest tiles of the shortest request.  Tile number idx is found without sorting: T(w), the number of tiles of all
// requests whose key is >= w, falls with w, so a binary search finds the key of the request that owns it.
// tiles_of(r, key, nt) gives a request's key and number of tiles (0: it has none and its key is 0).
template <typename TilesOf>
__device__ __forceinline__ bool pick_longest_request_first(const BatchParams& bp, int idx, int lane, TilesOf tiles_of, int* r_out,
                                                           int* b_out) {
  auto tiles_ge = [&](int w) {
    int c = 0;
    for (int r = lane; r < bp.B; r += 32) {
      int key, nt;
      tiles_of(r, key, nt);
      c += key >= w ? nt : 0;
    }
#pragma unroll
    for (int sh = 16; sh; sh >>= 1) c += __shfl_xor_sync(0xffffffffu, c, sh);
    return c;
  };
  int w_max = 0;
  for (int r = lane; r < bp.B; r += 32) {
    int key, nt;
    tiles_of(r, key, nt);
    w_max = max(w_max, key);
  }
#pragma unroll
  for (int sh = 16; sh; sh >>= 1) w_max = max(w_max, __shfl_xor_sync(0xffffffffu, w_max, sh));
  if (tiles_ge(1) <= idx) return false;
  int lo = 1, hi = w_max + 1, above = 0;  // tiles_ge(lo) > idx >= tiles_ge(hi) = above
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    const int c = tiles_ge(mid);
    if (c > idx) {
      lo = mid;
    } else {
      hi = mid;
      above = c;
    }
  }
  int k = idx - above;  // tile index among the requests whose key is exactly lo, taken in ascending request order
  for (int base = 0; base < bp.B; base += 32) {
    const int r = base + lane;
    int key = 0, nt = 0;
    if (r < bp.B) tiles_of(r, key, nt);
    const int mine = key == lo ? nt : 0;
    int incl = mine;  // inclusive prefix sum over the lanes
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, incl, sh);
      if (lane >= sh) incl += v;
    }
    const int total = __shfl_sync(0xffffffffu, incl, 31);
    if (k < total) {
      const unsigned hit = __ballot_sync(0xffffffffu, mine > 0 && k >= incl - mine && k < incl);
      const int sel = __ffs(hit) - 1;
      const int before = __shfl_sync(0xffffffffu, incl - mine, sel), ntile = __shfl_sync(0xffffffffu, nt, sel);
      *r_out = base + sel;
      *b_out = ntile - 1 - (k - before);  // longest tile first
      return true;
    }
    k -= total;
  }
  return false;
}

}  // namespace hswa_dev
