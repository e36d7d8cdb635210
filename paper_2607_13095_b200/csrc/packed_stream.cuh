// What the kernels for few rows over a 4-bit cache share: the sequence of key tiles, its cut into runs, the fragments' key order.
#pragma once

#include "packed.cuh"

namespace hswa_dev {

constexpr int kStreamTile = 64;  // keys per tile of the warp-level kernels

// Keys of a 16-key group in the order of the fragments' rows: row i of the first half holds key key_of(i), row 8 + i key 8 +
// key_of(i).  (A lane's V rows are key_of(2t), key_of(2t + 1): this order has lanes t = 0 .. 3 on rows 0, 3, 4, 7 and 1, 2, 5, 6,
// two of each parity, which halves the bank conflicts of 64-byte rows; K rows come in pairs of unlike parity.)
__device__ __forceinline__ int key_of(int i) { return (i & 4) | ((i & 2) ? 3 - (i & 1) : (i & 1)); }

// Keys of request r that the rows of a step see, and its tiles (one at least, if it has rows: zeros are written there too).
struct Stream {
  int t0, n, len, end, tiles;
};
template <int TILE = kStreamTile>
__device__ __forceinline__ Stream stream_of(const PackedAttnParams& p, int r) {
  Stream s;
  s.t0 = p.b.q_indptr ? p.b.q_indptr[r] : r;
  s.n = p.b.q_indptr ? min(p.b.q_indptr[r + 1] - s.t0, p.max_q_len) : 1;
  s.len = max(0, min(p.b.ctx_len[r], p.max_ctx_len));
  const int64_t room = (int64_t)p.b.max_blocks * p.m.P;  // positions that the block table has places for
  s.end = (int)min((int64_t)(p.causal ? s.len + s.n : s.len), room);
  s.tiles = s.n > 0 ? max(1, (s.end + TILE - 1) / TILE) : 0;
  return s;
}
// First tile of run c of `runs` over `total` tiles.
__device__ __forceinline__ int64_t run_start(int64_t total, int c, int runs) { return total * c / runs; }

// The requests' tiles summed by a block of THREADS threads: all tiles of one KV head, and this thread's first request i0, last i1
// and the tiles before i0.  s_sums: [THREADS / 32].
template <int THREADS, int TILE = kStreamTile>
__device__ __forceinline__ int64_t sum_tiles(const PackedAttnParams& p, int64_t* s_sums, int* i0, int* i1, int64_t* before) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, B = p.b.B, per = (B + THREADS - 1) / THREADS;
  *i0 = min((int)threadIdx.x * per, B);
  *i1 = min(*i0 + per, B);
  int64_t mine = 0;
  for (int i = *i0; i < *i1; ++i) mine += stream_of<TILE>(p, i).tiles;
  int64_t incl = mine;
#pragma unroll
  for (int sh = 1; sh < 32; sh <<= 1) {
    const int64_t v = __shfl_up_sync(0xffffffffu, incl, sh);
    if (lane >= sh) incl += v;
  }
  if (lane == 31) s_sums[warp] = incl;
  __syncthreads();
  int64_t total = 0;
  *before = incl - mine;
  for (int w = 0; w < THREADS / 32; ++w) {
    if (w < warp) *before += s_sums[w];
    total += s_sums[w];
  }
  return total;
}

// What the host's bounds do not cover of the batch is recorded (by one block of `threads` threads).
__device__ __forceinline__ void record_batch(const PackedAttnParams& p, int threads) {
  for (int r = threadIdx.x; r < p.b.B; r += threads) {
    const int ctx = p.b.ctx_len[r], t0 = p.b.q_indptr ? p.b.q_indptr[r] : r, n = p.b.q_indptr ? p.b.q_indptr[r + 1] - t0 : 1;
    const Stream s = stream_of(p, r);
    if (ctx < 0 || ctx > p.max_ctx_len) record_error(p.err, HSWA_ERR_BOUNDS, r, -1, ctx);
    if (n < 0 || n > p.max_q_len || t0 < 0 || (int64_t)t0 + n > p.total_q) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, n);
    if (p.causal && s.n > 0 && s.end < s.len + s.n) record_error(p.err, HSWA_ERR_BOUNDS, r, -3, s.len + s.n);
  }
}

}  // namespace hswa_dev
