// Eviction from a Full layer's cache by accumulated attention weight: the choice of the positions that stay, and their move
// to the head of fresh pages (paper Sec. 3.1.3: pages may be shared between requests, so kept rows are copied to pages of
// the request's own, never moved inside pages that another one reads).
#include "hswa_internal.cuh"

namespace {
using namespace hswa_dev;

// ---------------------------------------------------------------------------------------------------------------------
// Order-preserving map of a weight to 32 bits: NaN lowest, -0 and +0 alike, protected positions above everything.
__device__ __forceinline__ uint32_t rank_key(float w, int j, int ctx, int first, int last) {
  if (j < first || j >= ctx - last) return 0xffffffffu;
  if (w != w) return 0u;
  if (w == 0.f) return 0x80000000u;
  const uint32_t u = __float_as_uint(w);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The choice for one row (request, KV head), by one block.  The threshold, the keep-th largest key, is narrowed down by
// counting keys in bins.
//
// Counting every key of a long row in shared memory would cost more than reading it (an atomic per key, several keys of a
// warp in one bin), so long rows are sampled first: eight keys per thread, spread over the row, say below which key nothing
// can matter, with a margin of three standard deviations and more.  One pass then collects the keys from that one on in shared memory,
// in any order (warps do not wait for one another), and the threshold is found among them: the weights are read once.  The
// sample decides nothing: when the list turns out to hold fewer keys than are to stay, or does not fit, and on short rows,
// the top digit is counted over the whole row and the list begins at the digit found.  What stays is marked in a bitmap of
// the positions, which puts it in order.  A list that does not fit even then (many equal weights) is done without: the
// later passes read the row.
//
// Bound by what one SM can load -- a row is one block's -- and by the chain of block-wide steps around it.  512 rows of 1024
// to 32768 weights: 44 us for 41 MB (36 where launch follows launch); 128 rows of 65536 to 262144: 53 us for 83 MB, of which
// the longest row's 1 MB takes 32 us.
constexpr int SEL_BINS = 2048;
constexpr int SEL_QUADS = 4;  // quads of keys a thread has in hand in a step of the whole block

// Counters of a block-wide step.
template <int T>
struct SelectShared {
  uint32_t hist[SEL_BINS];
  uint32_t warp_sum[2][T / 32];   // packed counts per warp, two buffers in turn
  uint32_t warp_sum2[2][T / 32];
  uint32_t digit, want, n_list, n_near;
  uint32_t near[T];               // the keys that share the threshold's bin, when they are few, and their positions
  int near_pos[T], last;
};

// Position of a block-wide ordered step: thread-order prefix sums of four counts per thread (each at most 4), tile by tile.
// In: c = the counts of tiles 0..3 in bytes.  Out: per tile the sum over all threads before this one, tile 0's threads
// first; returns the grand total.  One barrier; `turn` alternates.
template <int T>
__device__ __forceinline__ uint32_t block_offsets(uint32_t (&sums)[2][T / 32], int turn, uint32_t c, uint32_t (&at)[SEL_QUADS]) {
  constexpr int NW = T / 32;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t incl = c;  // a warp's byte sums are at most 128
#pragma unroll
  for (int sh = 1; sh < 32; sh <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, sh);
    if (lane >= sh) incl += v;
  }
  if (lane == 31) sums[turn][warp] = incl;
  __syncthreads();
  const uint32_t w = lane < NW ? sums[turn][lane] : 0u;
  uint32_t even = w & 0x00ff00ffu, odd = (w >> 8) & 0x00ff00ffu;  // 16 bits each: at most 4096
#pragma unroll
  for (int sh = 1; sh < 32; sh <<= 1) {
    const uint32_t a = __shfl_up_sync(0xffffffffu, even, sh), b = __shfl_up_sync(0xffffffffu, odd, sh);
    if (lane >= sh) {
      even += a;
      odd += b;
    }
  }
  const uint32_t te = __shfl_sync(0xffffffffu, even, 31), to = __shfl_sync(0xffffffffu, odd, 31);
  uint32_t be = __shfl_sync(0xffffffffu, even, warp > 0 ? warp - 1 : 0), bo = __shfl_sync(0xffffffffu, odd, warp > 0 ? warp - 1 : 0);
  if (warp == 0) be = bo = 0;
  const uint32_t mine = incl - c;
  const uint32_t t0 = te & 0xffff, t1 = to & 0xffff, t2 = te >> 16, t3 = to >> 16;
  at[0] = (be & 0xffff) + (mine & 0xff);
  at[1] = t0 + (bo & 0xffff) + ((mine >> 8) & 0xff);
  at[2] = t0 + t1 + (be >> 16) + ((mine >> 16) & 0xff);
  at[3] = t0 + t1 + t2 + (bo >> 16) + (mine >> 24);
  return t0 + t1 + t2 + t3;
}

// Place of word i of a bitmap: one word of padding per 32, so that threads with consecutive words meet no bank twice.
__host__ __device__ __forceinline__ int map_at(int i) { return i + (i >> 5); }

// Lane i holds warp i's sum: the sum over the warps before this one.
__device__ __forceinline__ uint32_t sum_of_warps_before(uint32_t v) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  return __reduce_add_sync(0xffffffffu, lane < warp ? v : 0u);
}

// The highest digit at which the count from the top reaches `want`; `want` becomes the rank inside it.
template <int T>
__device__ __forceinline__ uint32_t find_digit(SelectShared<T>& sh, int bins, uint32_t& want) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr int PER = SEL_BINS / T;  // bins per thread, from the top down
  const int top = bins - 1 - (int)threadIdx.x * PER;
  uint32_t mine[PER], sum = 0;
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    mine[u] = top - u >= 0 ? sh.hist[top - u] : 0u;
    sum += mine[u];
  }
  uint32_t incl = sum;
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, s);
    if (lane >= s) incl += v;
  }
  if (lane == 31) sh.warp_sum[0][warp] = incl;
  __syncthreads();
  uint32_t b = incl - sum + sum_of_warps_before(lane < T / 32 ? sh.warp_sum[0][lane] : 0u);
#pragma unroll
  for (int u = 0; u < PER; ++u) {
    if (want > b && want <= b + mine[u]) {
      sh.digit = (uint32_t)(top - u);
      sh.want = want - b;
    }
    b += mine[u];
  }
  __syncthreads();
  want = sh.want;
  return sh.digit;
}

// Of the sample's keys, `share` should be among those that stay: the rank in the sample of a key that is below the threshold.
__host__ __device__ __forceinline__ float sample_rank(float share) { return share + 3.f * sqrtf(share) + 8.f; }

// T threads; CQ quads of keys per thread in flight while as many are looked at.
template <int T, int CQ>
__global__ void __launch_bounds__(T, T == 256 ? 4 : CQ == 4 ? 2 : 1) evict_select_kernel(const SelectParams p, const int capacity, const int words) {
  extern __shared__ __align__(16) uint32_t list[];  // [capacity] keys, [capacity] positions, [2] padded arrays of `words`
  __shared__ SelectShared<T> sh;
  const int row = blockIdx.x, kh = row % p.Hkv, r = row / p.Hkv;
  const int tid = threadIdx.x;
  int ctx = p.ctx_len[r];
  int keep = p.keep_len[r];
  if (ctx < 0 || ctx > p.max_ctx_len || keep < 0 || keep > p.max_keep) {
    if (tid == 0 && kh == 0)
      record_error(p.err, HSWA_ERR_BOUNDS, r, ctx < 0 || ctx > p.max_ctx_len ? -1 : -2, ctx < 0 || ctx > p.max_ctx_len ? ctx : keep);
    ctx = max(0, min(ctx, p.max_ctx_len));
    keep = max(0, min(keep, p.max_keep));
  }
  keep = min(keep, ctx);
  const float* w = p.weights + (int64_t)row * p.stride;
  int32_t* out = p.keep_idx + (int64_t)row * p.max_keep;
  if (tid == 0 && kh == 0) p.kept_len[r] = keep;
  for (int i = keep + tid; i < p.max_keep; i += T) out[i] = -1;
  if (keep == 0) return;
  if (keep == ctx) {  // everything stays
    for (int i = tid; i < keep; i += T) out[i] = i;
    return;
  }

  // The row in quads on 16-byte boundaries; the first one may begin up to three places before the row
  const int mis = (int)((reinterpret_cast<uintptr_t>(w) >> 2) & 3);
  const int quads = (ctx + mis + 3) / 4;
  auto quad_inside = [&](int q) {  // which of a quad's four places lie in the row
    const int j = q * 4 - mis;
    uint32_t in = 15u;
    if (j < 0) in &= 15u << -j;
    if (j + 4 > ctx) in &= 15u >> (j + 4 - ctx);
    return in;
  };
  auto load_quad = [&](int q) {
    const int j = q * 4 - mis;
    if (j >= 0 && j + 4 <= ctx) return __ldg(reinterpret_cast<const float4*>(w + j));
    float4 v;
    v.x = j >= 0 ? w[j] : 0.f;  // (the row is not empty, and a quad holds at least one place of it)
    v.y = j + 1 >= 0 && j + 1 < ctx ? w[j + 1] : 0.f;
    v.z = j + 2 >= 0 && j + 2 < ctx ? w[j + 2] : 0.f;
    v.w = j + 3 >= 0 && j + 3 < ctx ? w[j + 3] : 0.f;
    return v;
  };
  auto keys_of = [&](const float4& v, int q, uint32_t (&k)[4]) {
    const int j = q * 4 - mis;
    k[0] = rank_key(v.x, j, ctx, p.protect_first, p.protect_last);
    k[1] = rank_key(v.y, j + 1, ctx, p.protect_first, p.protect_last);
    k[2] = rank_key(v.z, j + 2, ctx, p.protect_first, p.protect_last);
    k[3] = rank_key(v.w, j + 3, ctx, p.protect_first, p.protect_last);
  };

  uint32_t* l_key = list;
  int32_t* l_pos = reinterpret_cast<int32_t*>(list + capacity);
  int turn = 0;
  uint32_t* map = list + 2 * capacity;                // the positions that stay, a bit each
  uint32_t* map_before = map + map_at(words);         // how many come before a word's
  const int lane = tid & 31;
  // Keys from `least_key` on, and their positions, into the list as far as they fit; returns their number.
  auto collect = [&](uint32_t least_key) {
    // The key as a weight: from zero on one comparison per weight says the same (a NaN compares false, and its key is 0).
    // Protected places, and rows whose list begins among negative weights, take the long way.
    const float least = __uint_as_float(least_key & 0x7fffffffu);
    const bool plain = least_key >= 0x80000000u;
    if (tid == 0) sh.n_list = 0;
    __syncthreads();
    // Quads [q_in, q_out) lie in the row and hold no protected place; a warp's round is mostly made of such.
    const int q_in = (min(max(p.protect_first, 0), ctx) + mis + 3) / 4;
    const int q_out = max(0, ctx - min(p.protect_last, ctx) + mis) / 4;
    const float4* row4 = reinterpret_cast<const float4*>(w - mis);
    auto all_in = [&](int q0) { return q0 >= q_in && q0 + (CQ - 1) * T + 32 <= q_out; };
    float4 v[CQ];
    auto fetch = [&](int q0) {
      if (all_in(q0)) {
#pragma unroll
        for (int u = 0; u < CQ; ++u) v[u] = __ldg(row4 + q0 + u * T + lane);
      } else {
#pragma unroll
        for (int u = 0; u < CQ; ++u)
          if (q0 + u * T + lane < quads) v[u] = load_quad(q0 + u * T + lane);
      }
    };
    fetch(tid - lane);
    for (int q0 = tid - lane; q0 < quads; q0 += CQ * T) {  // (the same for the lanes of a warp)
      float4 x[CQ];
#pragma unroll
      for (int u = 0; u < CQ; ++u) x[u] = v[u];
      fetch(q0 + CQ * T);  // the next round's loads are under way meanwhile
      uint32_t take = 0;   // four bits per quad
      if (plain && all_in(q0)) {
#pragma unroll
        for (int u = 0; u < CQ; ++u)
          take |= (x[u].x >= least ? 1u << (4 * u) : 0u) | (x[u].y >= least ? 2u << (4 * u) : 0u) |
                  (x[u].z >= least ? 4u << (4 * u) : 0u) | (x[u].w >= least ? 8u << (4 * u) : 0u);
      } else {
#pragma unroll 1
        for (int u = 0; u < CQ; ++u) {
          const int q = q0 + u * T + lane;
          if (q >= quads) break;
          uint32_t k[4], t = 0;
          keys_of(load_quad(q), q, k);  // (loaded again: this is the row's two ends)
#pragma unroll
          for (int e = 0; e < 4; ++e) t |= (k[e] >= least_key ? 1u : 0u) << e;
          take |= (t & quad_inside(q)) << (4 * u);
        }
        __syncwarp();
      }
      if (!__any_sync(0xffffffffu, take != 0)) continue;
      const uint32_t mine = __popc(take);
      uint32_t incl = mine;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += y;
      }
      uint32_t base = 0;
      if (lane == 31 && incl > 0) base = atomicAdd(&sh.n_list, incl);
      uint32_t slot = __shfl_sync(0xffffffffu, base, 31) + incl - mine;
      for (uint32_t m = take; m != 0; m &= m - 1, ++slot) {
        const int b = __ffs(m) - 1;
        if (slot < (uint32_t)capacity) l_pos[slot] = (q0 + (b >> 2) * T + lane) * 4 - mis + (b & 3);
      }
    }
    __syncthreads();
    const uint32_t n = sh.n_list;
    // the keys, read again (from L2) for the few that are listed: four at a time
    const int n_in = (int)min(n, (uint32_t)capacity);
    for (int i0 = tid; i0 < n_in; i0 += 4 * T) {
      float x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) x[u] = i0 + u * T < n_in ? __ldg(w + l_pos[i0 + u * T]) : 0.f;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * T < n_in) l_key[i0 + u * T] = rank_key(x[u], l_pos[i0 + u * T], ctx, p.protect_first, p.protect_last);
    }
    __syncthreads();
    return n;
  };
  auto clear_hist = [&]() {
    for (int i = tid; i < SEL_BINS; i += T) sh.hist[i] = 0;
    __syncthreads();
  };

  uint32_t want = (uint32_t)keep, n_list = 0;
  bool listed = false;
  // The threshold is at least `low`, and below low + 2^bits (bits = 32: anywhere from low on); `want` of the keys in that
  // range stay, and all keys above it.
  uint32_t low = 0;
  int bits = 32;
  // ---- long rows: a sample's word on where the list may begin ----
  if (quads >= 4 * T) {
    const int step = quads / (2 * T);
    const float share = 8.f * T * (float)keep / (float)ctx;  // of the sample's 8 T keys, those that would stay
    uint32_t rank = (uint32_t)sample_rank(share);
    if (rank <= 4 * T) {  // at most half of it
      uint32_t k[2][4], in[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int q = (u * T + tid) * step + step / 2;
        keys_of(load_quad(q), q, k[u]);
        in[u] = quad_inside(q);
      }
#pragma unroll
      for (int digit = 0; digit < 2; ++digit) {  // 22 bits of it
        clear_hist();
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (((in[u] >> e) & 1u) && (digit == 0 || (k[u][e] >> 21) == (low >> 21)))
              atomicAdd(&sh.hist[digit == 0 ? k[u][e] >> 21 : (k[u][e] >> 10) & 2047u], 1u);
        __syncthreads();
        low |= find_digit<T>(sh, SEL_BINS, rank) << (digit == 0 ? 21 : 10);
      }
      n_list = collect(low);
      listed = n_list >= (uint32_t)keep && n_list <= (uint32_t)capacity;
    }
  }
  // ---- the top digit, counted over the row ----
  if (!listed) {
    clear_hist();
    for (int q0 = tid; q0 < quads; q0 += SEL_QUADS * T) {
      float4 v[SEL_QUADS];
#pragma unroll
      for (int u = 0; u < SEL_QUADS; ++u)
        if (q0 + u * T < quads) v[u] = load_quad(q0 + u * T);
#pragma unroll
      for (int u = 0; u < SEL_QUADS; ++u) {
        const int q = q0 + u * T;
        if (q < quads) {
          uint32_t k[4];
          keys_of(v[u], q, k);
          const uint32_t in = quad_inside(q);
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if ((in >> e) & 1u) atomicAdd(&sh.hist[k[e] >> 21], 1u);
        }
      }
    }
    __syncthreads();
    const uint32_t d1 = find_digit<T>(sh, SEL_BINS, want);
    low = d1 << 21;
    bits = 21;
    n_list = (uint32_t)keep - want + sh.hist[d1];  // keys above the digit, and all that have it
    listed = n_list <= (uint32_t)capacity;
    __syncthreads();  // everybody has read the bin
    if (listed) collect(low);
  }

  // ---- the threshold: narrowed down over the list or over the row ----
  const int n_quads = listed ? (int)(n_list + 3) / 4 : quads;
  auto get = [&](int q, uint32_t (&k)[4]) -> uint32_t {  // a quad's keys; which of its places count
    if (listed) {
      const uint4 v = reinterpret_cast<const uint4*>(l_key)[q];  // (the list's room is whole quads)
      k[0] = v.x;
      k[1] = v.y;
      k[2] = v.z;
      k[3] = v.w;
      return q * 4 + 4 <= (int)n_list ? 15u : 15u >> (q * 4 + 4 - (int)n_list);
    }
    keys_of(load_quad(q), q, k);
    return quad_inside(q);
  };
  // One step: the bin of 2^shift keys that holds the threshold; false if that is the last bin of a range cut off at 2^32
  // keys, which also holds everything beyond.
  // by_pos: among the listed keys equal to `thr`, the same for their positions from the lowest on (as their complements).
  uint32_t thr = 0;
  auto narrow = [&](int shift, bool by_pos) {
    const int bins = bits == 32 ? SEL_BINS : 1 << (bits - shift);
    clear_hist();
    for (int q = tid; q < n_quads; q += T) {
      uint32_t k[4];
      uint32_t in = get(q, k);
      if (by_pos) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (k[e] != thr) in &= ~(1u << e);
          k[e] = ~(uint32_t)l_pos[q * 4 + e];
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t b = k[e] >= low ? (k[e] - low) >> shift : 0xffffffffu;
        if (((in >> e) & 1u) && k[e] >= low && (bits == 32 || b < (uint32_t)bins)) atomicAdd(&sh.hist[min(b, (uint32_t)bins - 1u)], 1u);
      }
    }
    __syncthreads();
    uint32_t rank = want;
    const uint32_t d = find_digit<T>(sh, bins, rank);
    if (bits == 32 && shift < 21 && d == (uint32_t)bins - 1u) return false;
    want = rank;
    low += d << shift;
    bits = shift;
    return true;
  };
  if (bits == 32) {
    // A list from `low` on: bins of 2^16 keys (1/128 of an octave) over 16 octaves tell most apart and keep the keys of a
    // warp out of one bin; if the threshold lies beyond, bins of whole digits.
    if (!narrow(16, false)) {
      low = 0;
      narrow(21, false);
    }
  }
  int last_tie = -1;  // listed: of the keys equal to the threshold, those up to this position stay
  while (bits > 0) {
    const uint32_t near = sh.hist[sh.digit];  // (as the last step, or the count of the top digit, left them)
    __syncthreads();
    if (near > (uint32_t)T) {
      narrow(bits > 11 ? bits - 11 : 0, false);
      continue;
    }
    // few keys share the bin: each is ranked among them, equal ones by position
    if (tid == 0) sh.n_near = 0;
    __syncthreads();
    for (int q = tid; q < n_quads; q += T) {
      uint32_t k[4];
      const uint32_t in = get(q, k);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (((in >> e) & 1u) && k[e] >= low && ((k[e] - low) >> bits) == 0) {
          const uint32_t at = atomicAdd(&sh.n_near, 1u);
          if (at < (uint32_t)T) {
            sh.near[at] = k[e];
            sh.near_pos[at] = listed ? l_pos[q * 4 + e] : q * 4 - mis + e;
          }
        }
    }
    __syncthreads();
    if (tid < (int)near) {
      const uint32_t k = sh.near[tid];
      const int pos = sh.near_pos[tid];
      uint32_t above = 0, before = 0;  // larger keys; equal ones at lower positions
      for (int i = 0; i < (int)near; ++i) {
        above += sh.near[i] > k;
        before += sh.near[i] == k && sh.near_pos[i] < pos;
      }
      if (above + before == want - 1) {  // the last one that stays
        sh.digit = k;
        sh.want = before + 1;
        sh.last = pos;
      }
    }
    __syncthreads();
    low = sh.digit;
    want = sh.want;
    last_tie = sh.last;
    break;
  }
  thr = low;
  if (listed && bits == 0) {  // many equal keys
    low = 0;
    bits = 32;
    narrow(21, true);
    narrow(10, true);
    narrow(0, true);
    last_tie = (int)~low;
  }

  // ---- the kept positions: keys above the threshold, and the first `want` of those equal to it ----
  if (listed) {
    uint32_t done = 0;
    int32_t* in_order = reinterpret_cast<int32_t*>(l_key);  // [keep]: written when the keys have been looked at
    const bool windows = ctx > words * 32;
    auto stays = [&](int i) { return l_key[i] > thr || (l_key[i] == thr && l_pos[i] <= last_tie); };
    if (windows) {  // the list is gone through more than once: what goes loses its position
      for (int i = tid; i < (int)n_list; i += T)
        if (!stays(i)) l_pos[i] = -1;
    }
    for (int win = 0; win < ctx; win += words * 32) {  // positions a bitmap at a time
      const int n_words = min(words, (ctx - win + 31) / 32), each = (n_words + T - 1) / T;
      for (int i = tid; i < map_at(n_words); i += T) map[i] = 0;
      __syncthreads();
      for (int i = tid; i < (int)n_list; i += T) {
        const int j = l_pos[i] - win;
        if (j >= 0 && j < n_words * 32 && (windows || stays(i))) atomicOr(map + map_at(j >> 5), 1u << (j & 31));
      }
      __syncthreads();
      // a thread counts consecutive words
      const int w_lo = min(tid * each, n_words), w_hi = min(w_lo + each, n_words);
      uint32_t c = 0;
      for (int i = w_lo; i < w_hi; ++i) c += __popc(map[map_at(i)]);
      uint32_t incl = c;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, incl, d);
        if (lane >= d) incl += x;
      }
      if (lane == 31) sh.warp_sum[0][tid >> 5] = incl;
      __syncthreads();
      const uint32_t of_warp = lane < T / 32 ? sh.warp_sum[0][lane] : 0u;
      uint32_t at = done + incl - c + sum_of_warps_before(of_warp);
      done += __reduce_add_sync(0xffffffffu, of_warp);
      for (int i = w_lo; i < w_hi; ++i) {
        map_before[map_at(i)] = at;
        at += __popc(map[map_at(i)]);
      }
      __syncthreads();
      for (int i = tid; i < n_words; i += T) {  // full words next to one another fall to different threads
        uint32_t slot = map_before[map_at(i)];
        for (uint32_t m = map[map_at(i)]; m != 0; m &= m - 1, ++slot)
          if (slot < (uint32_t)keep) in_order[slot] = win + i * 32 + __ffs(m) - 1;
      }
      __syncthreads();
    }
    for (int i = tid; i < keep; i += T) out[i] = in_order[i];
    return;
  }
  uint32_t base_gt = 0, base_eq = 0;
  for (int q0 = 0; q0 < n_quads; q0 += SEL_QUADS * T) {
    uint32_t gt[SEL_QUADS], eq[SEL_QUADS], c_gt = 0, c_eq = 0;
#pragma unroll
    for (int u = 0; u < SEL_QUADS; ++u) {
      const int q = q0 + u * T + tid;
      gt[u] = eq[u] = 0;
      if (q < n_quads) {
        uint32_t k[4];
        const uint32_t in = get(q, k);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          gt[u] |= (k[e] > thr ? 1u : 0u) << e;
          eq[u] |= (k[e] == thr ? 1u : 0u) << e;
        }
        gt[u] &= in;
        eq[u] &= in;
      }
      c_gt |= (uint32_t)__popc(gt[u]) << (8 * u);
      c_eq |= (uint32_t)__popc(eq[u]) << (8 * u);
    }
    uint32_t at_gt[SEL_QUADS], at_eq[SEL_QUADS];
    const uint32_t all_gt = block_offsets<T>(sh.warp_sum, turn, c_gt, at_gt);
    const uint32_t all_eq = block_offsets<T>(sh.warp_sum2, turn, c_eq, at_eq);
    turn ^= 1;
#pragma unroll
    for (int u = 0; u < SEL_QUADS; ++u) {
      uint32_t g = base_gt + at_gt[u], e_rank = base_eq + at_eq[u];
      const int q = q0 + u * T + tid;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool is_gt = (gt[u] >> e) & 1u, is_eq = (eq[u] >> e) & 1u;
        const uint32_t slot = g + min(e_rank, want);
        if ((is_gt || (is_eq && e_rank < want)) && slot < (uint32_t)keep) out[slot] = q * 4 - mis + e;
        g += is_gt;
        e_rank += is_eq;
      }
    }
    base_gt += all_gt;
    base_eq += all_eq;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Kept row i of (request, KV head) goes from the storage of position keep_idx[i] to that of position i behind the new
// block table.  A warp takes `rows` consecutive kept rows: lane l looks up row l's source and destination, then the warp
// copies the rows with 16 bytes per lane, eight loads in flight before the first store.  Bound by memory: 2 x 4 D bytes per
// row (source rows are gathered 2 D bytes at a time, destinations are consecutive).  32 requests, 8 heads of 128, 4096 of up to
// 16384 rows kept: 162 us for 0.99 GB = 6.1 TB/s (one row per warp: 429 us).
template <int D>
__global__ void __launch_bounds__(256) evict_compact_kernel(const CompactParams p, const int rows) {
  constexpr int LPR = D / 4;         // lanes per row: K and V, 16 bytes each
  constexpr int RPS = 32 / LPR;      // rows per step
  constexpr int STEPS = 8;
  const ModelParams& M = p.m;
  const int kh = blockIdx.y, r = blockIdx.z, lane = threadIdx.x & 31;
  const int i0 = (blockIdx.x * 8 + (threadIdx.x >> 5)) * rows;
  int kept = p.kept_len[r];
  if (kept < 0 || kept > p.max_keep) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && kh == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, kept);
    kept = min(kept, p.max_keep);
  }
  if (i0 >= kept) return;
  const int ctx = min(p.b.ctx_len[r], p.max_ctx_len);
  const int64_t pair = (int64_t)r * M.Hkv + kh;
  const int i = i0 + lane;
  int64_t src = -1, dst = -1;  // element offsets of the K rows; -1: nothing to copy
  if (lane < rows && i < kept) {
    const int j = p.keep_idx[pair * p.max_keep + i];
    if (j < 0 || j >= ctx) {
      record_error(p.err, HSWA_ERR_BOUNDS, r, i, j);
    } else {
      const int from = p.b.block_table[(int64_t)r * p.b.max_blocks + j / M.P];
      const int to = p.dst_block_table[(int64_t)r * p.dst_max_blocks + i / M.P];
      if (from < 0 || from >= p.num_pages || to < 0 || to >= p.num_pages) {
        record_error(p.err, HSWA_ERR_BOUNDS, r, i, from < 0 || from >= p.num_pages ? from : to);
      } else {
        src = (((int64_t)from * 2 * M.Hkv + kh) * M.P + j % M.P) * D;
        dst = (((int64_t)to * 2 * M.Hkv + kh) * M.P + i % M.P) * D;
        if (p.weights) p.weights_out[pair * p.out_stride + i] = p.weights[pair * p.stride + j];
      }
    }
  }
  // K in the lower half of a row's lanes, V (Hkv * P rows further on) in the upper half
  const int64_t mine = (int64_t)(lane % LPR / (LPR / 2)) * M.Hkv * M.P * D + lane % (LPR / 2) * 8;
  for (int l0 = 0; l0 < rows; l0 += STEPS * RPS) {
    uint4 v[STEPS];
    int64_t to[STEPS];
#pragma unroll
    for (int u = 0; u < STEPS; ++u) {
      const int l = l0 + u * RPS + lane / LPR;  // the lane that looked this row up (rows is a multiple of STEPS * RPS)
      const int64_t from = __shfl_sync(0xffffffffu, src, l);
      to[u] = __shfl_sync(0xffffffffu, dst, l);
      if (from >= 0) v[u] = __ldcs(reinterpret_cast<const uint4*>(p.pool + from + mine));
    }
#pragma unroll
    for (int u = 0; u < STEPS; ++u)
      if (to[u] >= 0) *reinterpret_cast<uint4*>(p.pool + to[u] + mine) = v[u];
  }
}

}  // namespace

namespace {
// Shared memory of a block: the list and the bitmap of positions with a number per word.
struct SelectRoom {
  int capacity, words;
  int bytes() const { return (capacity + map_at(words)) * 8; }
};

// Room in the list for what stays and for what the threshold's bin brings with it, and for what a sample of 8 T keys brings
// with it when its rank is four standard deviations off.  A list that does not fit costs passes over the row: more room than
// leaves L1 its own is taken only for that (64 rows of 65536 to 262144, 16000 kept: 75 us; at 18432 places 312).
SelectRoom select_room(const SelectParams& p, int T) {
  SelectRoom room;
  const float share = 8.f * T * (float)p.max_keep / (float)(p.max_ctx_len > 0 ? p.max_ctx_len : 1), rank = sample_rank(share);
  int64_t capacity = (int64_t)p.max_keep + p.max_keep / 2 + (T == 512 ? 2048 : 1024);
  const int64_t sampled = (int64_t)((rank + 4.f * sqrtf(rank)) * (float)p.max_ctx_len / (8.f * T));
  if (capacity > 18432) capacity = 18432;  // (L1 keeps enough room for loads in flight)
  if (rank <= 4 * T && capacity < sampled) capacity = sampled;
  if (capacity > p.max_ctx_len) capacity = p.max_ctx_len;
  room.words = (p.max_ctx_len + 31) / 32;
  if (room.words > 4096) room.words = 4096;
  const int64_t most = (227 * 1024 - (int)sizeof(SelectShared<512>) - 64) / 8 - map_at(room.words) - 4;
  if (capacity > most) capacity = most;
  room.capacity = (int)((capacity + 3) / 4 * 4);
  return room;
}

template <int T, int CQ>
cudaError_t launch_select_t(const SelectParams& p, int64_t rows, cudaStream_t s) {
  const SelectRoom room = select_room(p, T);
  cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<T, CQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, room.bytes());
  if (e != cudaSuccess) return e;
  evict_select_kernel<T, CQ><<<(unsigned)rows, T, room.bytes(), s>>>(p, room.capacity, room.words);
  return cudaGetLastError();
}
}  // namespace

cudaError_t hswa_launch_evict_select(const SelectParams& p, int num_sms, cudaStream_t s) {
  if (p.B == 0) return cudaSuccess;
  const int64_t rows = (int64_t)p.B * p.Hkv;
  // Blocks.  More rows than SMs, up to 32768 positions: four small blocks per SM, whose steps overlap (512 rows, 2048 kept, us
  // with four small / two larger blocks: rows of 1024 to 32768 40.4 / 42.9, 8000 to 30000 39.9 / 43.6; above the limit 1024 to
  // 33500 40.4 / 43.4, 1024 to 65536 57.3 / 53.2, 30000 to 65536 with 4096 kept 76 / 65; 256 rows of 4000 to 30000 22.3 / 20.2,
  // to 33500 22.8 / 20.5: fewer rows per SM would rather have the larger ones).  Else two blocks of 512 threads per SM, where their lists leave L1 the room that the data of
  // loads in flight needs (512 rows of 30000 to 60000, 4096 kept: 66 us; four small blocks 76, one block 99), or one where there
  // is one row per SM at most (128 rows of 16000 to 32000: 19 us; small blocks 25).  The longest rows and lists: one block per
  // SM with as many loads in flight as its registers hold (128 rows of 65536 to 262144, 8191 kept: 54 us; with half of them
  // in flight 59; with 213 KB of shared memory instead of 195 or less, so that L1 is short of room, 70).
  if (rows > num_sms && p.max_ctx_len <= 32768) return launch_select_t<256, 4>(p, rows, s);
  const bool two_fit = select_room(p, 512).bytes() + (int)sizeof(SelectShared<512>) <= 96 * 1024;
  if (rows > num_sms ? two_fit : p.max_ctx_len <= 131072) return launch_select_t<512, 4>(p, rows, s);
  return launch_select_t<512, 8>(p, rows, s);
}

cudaError_t hswa_launch_evict_compact(const CompactParams& p, int num_sms, cudaStream_t s) {
  if (p.b.B == 0 || p.max_keep == 0) return cudaSuccess;
  // 32 kept rows per warp, fewer while the warps do not fill the machine
  int rows = 32;
  const int least = p.m.D == 128 ? 8 : 16;
  while (rows > least && (int64_t)p.b.B * p.m.Hkv * ((p.max_keep + rows - 1) / rows) < 32LL * num_sms) rows /= 2;
  dim3 grid((p.max_keep + 8 * rows - 1) / (8 * rows), p.m.Hkv, p.b.B);
  if (p.m.D == 128)
    evict_compact_kernel<128><<<grid, 256, 0, s>>>(p, rows);
  else
    evict_compact_kernel<64><<<grid, 256, 0, s>>>(p, rows);
  return cudaGetLastError();
}
