// Accumulated attention weights of the cached keys (hswa_attn_weights): weights[j] = decay * weights[j] + the sum over the
// step's rows (token, head of the group) of exp(scale q.k_j - lse), for every (request, KV head).
//
// A score product whose output is summed over its ROWS: keys are the M dimension of tcgen05.mma (128 keys = 128 TMEM lanes
// = 128 threads), the packed (token, head) rows are N, so that a thread owns a key, adds up its row sums in registers and
// writes one number.  With more than 64 rows a Q tile two threads own a key, each with one half of the columns, and their
// two sums meet through TMEM once per key tile.  No atomics, and the order of the sums is fixed.  Each key is read from
// memory once.
//
// Bounds.  One row group (a decode step) is bound by reading K: 64 requests of 4096 to 32768 keys, 8 KV heads of 128: 423 to
// 437 us = 6.3 to 6.5 TB/s, a plain copy's rate.  With many rows the sums bound it (an observation window of 33 to 64 tokens
// on 8 prompts of up to 16384: 74 us, where the tensor core has 26 us of work and the special-function units, at 16
// exponentials per clock and SM, 37 us; they are 61 % busy, the issue slots 43 %): the rest is the instructions and the waits
// around them.  Taking a share of the exponentials on the FMA pipes by a polynomial was slower (1, 2, 3 of 8: 78 us; 4 of 8:
// 83 us; none: 74).
//
// Warp roles: two groups of summing warps (four or eight each) take the even and the odd key tiles of a segment, one warp
// loads (TMA) and stages the rows' log-sum-exps, one issues the MMAs.  Each group has two TMEM accumulators.
//
// Blocks are persistent: all key tiles of the batch, weighted with the Q tiles they meet, are cut into equal shares, and a
// block walks the segments (request, KV head, range of key tiles) of its share with every pipeline running on across
// them.  The Q tiles of a segment (up to 128 rows each) stay in shared memory while it lasts when they all fit, else they
// are streamed from L2 once per pair of key tiles.
#include "hswa_internal.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int TKEYS = 128;       // keys per tile
// Summing warps per group: four cover the 128 keys of a tile.  The many-row form has twice as many, each with half of the
// columns: two warps per scheduler leave the pipes idle too long behind TMEM reads and dependent steps (86 us on an
// observation window of up to 64 tokens of 8 prompts of up to 16384, 78 us with four, both measured while three of eight
// exponentials were on the FMA pipes).
constexpr int group_warps(bool wide) { return wide ? 8 : 4; }
constexpr int block_threads(bool wide) { return (2 * group_warps(wide) + 2) * 32; }
constexpr int MAX_NSQ = 8, MAX_NSK = 6;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NO_ROW = -1e30f;  // in the place of an absent row's value, or of a row's that saw nothing: 2^that = 0

// Barriers
enum { B_QFULL = 0, B_LFULL = B_QFULL + MAX_NSQ, B_QEMPTY = B_LFULL + MAX_NSQ, B_KFULL = B_QEMPTY + MAX_NSQ,
       B_KEMPTY = B_KFULL + MAX_NSK, B_SFULL = B_KEMPTY + MAX_NSK /* [group][buffer] */, B_SEMPTY = B_SFULL + 4,
       B_PFULL = B_SEMPTY + 4 /* [group][buffer]: the upper columns' sums are in TMEM */, B_QLAND = B_PFULL + 4, NUM_BARS };

struct WeightsPlan {
  int n_cols;       // N of the MMA: rows of a Q tile, rounded up
  int tile_tokens;  // tokens per Q tile
  int nsq, nsk;     // Q and K stages
  int tmem_cols;
};

// Index of the error word for a request that the host's bounds, the block table or the weights do not cover; 0 if fine.
__device__ __forceinline__ int weights_request_error(const WeightsParams& p, int ctx, int t0, int n) {
  if (ctx < 0 || ctx > p.max_ctx_len) return -1;
  if (n < 0 || n > p.max_q_len || t0 < 0 || (int64_t)t0 + n > p.total_q) return -2;
  const int64_t keys = (int64_t)ctx + (p.causal ? n : 0);
  return keys > p.stride || keys > (int64_t)p.b.max_blocks * p.m.P ? -3 : 0;
}

// Columns that the MMA of a Q tile of `cols` rows writes, of the tile's N; those behind them hold what an earlier kernel or
// Q tile left in TMEM, and nothing may read them.
__device__ __forceinline__ int mma_cols(int cols, int N) { return min(N, (cols + 31) & ~31); }

// A warp's bounded wait: one answer for all lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

// One thread's sum over 16 score columns.  nl: minus the rows' log-sum-exps in log2 units; a column that does not count (an
// absent row) has NO_ROW there and a finite score.  MASKED: columns outside [c_lo, c_hi) are dropped whatever their score is.
template <bool MASKED>
__device__ __forceinline__ void sum_chunk(const uint32_t (&v)[16], const float* nl, float scale_log2, int c0, int c_lo, int c_hi,
                                          float2 (&acc)[4]) {
  const float2 sc2 = make_float2(scale_log2, scale_log2);
#pragma unroll
  for (int k = 0; k < 16; k += 4) {
    const float4 l4 = *reinterpret_cast<const float4*>(nl + k);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int c = k + 2 * h;
      const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[c]), __uint_as_float(v[c + 1])), sc2,
                                  h ? make_float2(l4.z, l4.w) : make_float2(l4.x, l4.y));
      float2 e = make_float2(fast_exp2(x.x), fast_exp2(x.y));
      if constexpr (MASKED) {
        e.x = c0 + c >= c_lo && c0 + c < c_hi ? e.x : 0.f;
        e.y = c0 + c + 1 >= c_lo && c0 + c + 1 < c_hi ? e.y : 0.f;
      }
      acc[(c >> 1) & 3] = __fadd2_rn(acc[(c >> 1) & 3], e);
    }
  }
}

// Position in a ring of stages: the slot, and the parity of the phase in which it is next filled.
struct Ring {
  int slot = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void step(int stages) {
    if (++slot == stages) {
      slot = 0;
      phase ^= 1u;
    }
  }
  __device__ __forceinline__ void step(int stages, int by) {  // by <= stages
    slot += by;
    if (slot >= stages) {
      slot -= stages;
      phase ^= 1u;
    }
  }
};

// A stretch of the block's share: key tiles [t_lo, t_hi) of one (request, KV head).
struct Segment {
  int r, kh, t0, n, ctx, kv_len, t_lo, t_hi, n_qt;
};

// Walks a block's share [lo, hi) of the batch's total cost.  A key tile costs, per Q tile of the request, four units
// and one more per 32 rows (measured: 0.83 us and 0.23 us per pair of key tiles); the first tile of a (request, KV head) costs
// three times that (its Q tiles come in, and the pipeline runs empty behind the segment before).  The tiles follow one another by
// KV head; a tile belongs to the share in which it begins.  Every role walks by itself.
struct Walker {
  int r;
  int64_t base, lo, hi;  // base: cost of all requests before r
  int kh;

  __device__ __forceinline__ static void request(const WeightsParams& p, const WeightsPlan& pl, int r, Segment& s, int& tiles, int& q) {
    s.r = r;
    s.t0 = p.b.q_indptr ? p.b.q_indptr[r] : r;
    s.n = p.b.q_indptr ? p.b.q_indptr[r + 1] - s.t0 : 1;
    s.ctx = p.b.ctx_len[r];
    tiles = 0;
    q = 1;
    if (weights_request_error(p, s.ctx, s.t0, s.n) != 0) return;
    s.kv_len = s.ctx + (p.causal ? s.n : 0);
    s.n_qt = (s.n + pl.tile_tokens - 1) / pl.tile_tokens;
    tiles = (s.kv_len + TKEYS - 1) / TKEYS;
    q = max(1, (s.n_qt - 1) * (4 + (pl.tile_tokens * p.m.G + 31) / 32) + 4 + ((s.n - (s.n_qt - 1) * pl.tile_tokens) * p.m.G + 31) / 32);
  }

  // Tiles of a (request, KV head) that begin before cost c of it: tile 0 at 0, tile i at (i + 2) q.
  __device__ __forceinline__ static int tiles_before(int64_t c, int tiles, int q) {
    if (c <= 0) return 0;
    const int64_t i = (c + q - 1) / q - 2;
    return (int)(i < 1 ? 1 : (i < tiles ? i : tiles));
  }

  __device__ __forceinline__ bool next(const WeightsParams& p, const WeightsPlan& pl, Segment& s) {
    for (; r < p.b.B && base < hi; ++r, kh = 0) {
      int tiles, q;
      request(p, pl, r, s, tiles, q);
      const int64_t head_cost = tiles > 0 ? (int64_t)(tiles + 2) * q : 0, all = head_cost * p.m.Hkv;
      if (lo < base + all) {
        if (lo > base + kh * head_cost) kh = (int)((lo - base) / head_cost);
        for (; kh < p.m.Hkv; ++kh) {
          const int64_t c0 = base + kh * head_cost;
          if (c0 >= hi) return false;
          s.t_lo = tiles_before(lo - c0, tiles, q);
          s.t_hi = tiles_before(hi - c0, tiles, q);
          if (s.t_lo < s.t_hi) {
            s.kh = kh++;
            return true;
          }
        }
      }
      base += all;
    }
    return false;
  }
};

// WIDE: one block per SM, Q tiles of up to 128 rows; else two blocks per SM (at most 64 rows).
template <int D, bool WIDE>
__global__ void __launch_bounds__(block_threads(WIDE), WIDE ? 1 : 2)
attn_weights_kernel(const __grid_constant__ CUtensorMap tm_pool, const __grid_constant__ CUtensorMap tm_q, const WeightsParams p,
                    const WeightsPlan pl) {
  constexpr int HALVES = D / 64;
  constexpr int K_HALF = TKEYS * 128, K_BYTES = HALVES * K_HALF;
  constexpr int GW = group_warps(WIDE), LOADER = 2 * GW, ISSUER = 2 * GW + 1, THREADS = block_threads(WIDE);
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int N = pl.n_cols;
  const uint32_t q_half = (uint32_t)N * 128, q_bytes = q_half * HALVES;
  const uint32_t off_k = pl.nsq * q_bytes, off_lse = off_k + pl.nsk * K_BYTES;
  float* s_nl = reinterpret_cast<float*>(smem + off_lse);                            // [nsq][N]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + off_lse + pl.nsq * N * 4);     // [NUM_BARS]
  int64_t* s_base = reinterpret_cast<int64_t*>(bars + NUM_BARS);                     // [2]: base and total
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(s_base + 2);
  int* s_r = reinterpret_cast<int*>(tmem_slot + 1);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  // ---- this block's share ----
  if (warp == 0) {
    auto cost_of = [&](int r) {
      if (r >= p.b.B) return (int64_t)0;
      Segment s;
      int tiles, q;
      Walker::request(p, pl, r, s, tiles, q);
      return tiles > 0 ? (int64_t)(tiles + 2) * q * M.Hkv : (int64_t)0;
    };
    int64_t total = 0;
    for (int r = lane; r < p.b.B; r += 32) total += cost_of(r);
#pragma unroll
    for (int sh = 16; sh; sh >>= 1) total += __shfl_xor_sync(0xffffffffu, total, sh);
    const int64_t lo = total * blockIdx.x / gridDim.x;
    int64_t base = 0;
    int at = p.b.B;
    for (int r0 = 0; r0 < p.b.B; r0 += 32) {
      const int64_t c = cost_of(r0 + lane);
      int64_t incl = c;
#pragma unroll
      for (int sh = 1; sh < 32; sh <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, incl, sh);
        if (lane >= sh) incl += v;
      }
      const unsigned hit = __ballot_sync(0xffffffffu, base + incl > lo);  // the first request whose tiles reach past lo
      if (hit) {
        const int sel = __ffs(hit) - 1;
        at = r0 + sel;
        base += __shfl_sync(0xffffffffu, incl - c, sel);
        break;
      }
      base += __shfl_sync(0xffffffffu, incl, 31);
    }
    if (lane == 0) {
      s_base[0] = base;
      s_base[1] = total;
      *s_r = at;
    }
  } else if (warp == 1 && blockIdx.x == 0) {
    for (int r = lane; r < p.b.B; r += 32) {
      const int t0 = p.b.q_indptr ? p.b.q_indptr[r] : r, n = p.b.q_indptr ? p.b.q_indptr[r + 1] - t0 : 1, ctx = p.b.ctx_len[r];
      const int bad = weights_request_error(p, ctx, t0, n);
      if (bad != 0) record_error(p.err, HSWA_ERR_BOUNDS, r, bad, bad == -1 ? ctx : bad == -2 ? n : ctx + n);
    }
  }
  if (threadIdx.x == 64) {
    for (int i = 0; i < pl.nsq; ++i) {
      mbar_init(bar(B_QFULL + i), 1);
      mbar_init(bar(B_LFULL + i), 1);
      mbar_init(bar(B_QEMPTY + i), 1 + 2 * GW);  // the MMA commit and the summing warps
    }
    for (int i = 0; i < pl.nsk; ++i) {
      mbar_init(bar(B_KFULL + i), 1);
      mbar_init(bar(B_KEMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_SEMPTY + i), GW);
      mbar_init(bar(B_PFULL + i), 4);
    }
    mbar_init(bar(B_QLAND), 1);
    mbar_fence_init();
    tma_prefetch_desc(&tm_pool);
    tma_prefetch_desc(&tm_q);
    if (sbase & 1023u) record_error(p.err, HSWA_ERR_CUDA, -1, (int)(sbase & 1023u), 16);  // tiles would be misread
  }
  // rows of a Q tile that no load fills (a group that does not divide the tile): zeros, so that their scores are finite
  const int q_rows = pl.tile_tokens * M.G;
  for (int i = threadIdx.x; i < pl.nsq * HALVES * (N - q_rows) * 8; i += THREADS) {
    const int ch = i & 7, row = q_rows + (i >> 3) % (N - q_rows), hs = (i >> 3) / (N - q_rows);
    *reinterpret_cast<uint4*>(smem + (hs / HALVES) * q_bytes + (hs % HALVES) * q_half + row * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  if (warp == ISSUER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(pl.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  Walker walk;
  walk.r = *s_r;
  walk.kh = 0;
  walk.base = s_base[0];
  walk.lo = s_base[1] * blockIdx.x / gridDim.x;
  walk.hi = s_base[1] * (blockIdx.x + 1) / gridDim.x;
  Segment sg;
  // first Q tile with a token that sees any key of tile t (causal: token i sees j <= ctx + i)
  auto first_qt = [&](int t) {
    const int over = t * TKEYS - sg.ctx;
    return p.causal && over > 0 ? over / pl.tile_tokens : 0;
  };

  if (warp == LOADER) {
    // ======================= loader =======================
    const int ppt = TKEYS / M.P;
    bool ok = true;
    int row_tok[4], row_at[4];  // of the lane's four rows of a Q tile: the token in the tile, the place of its log-sum-exp
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int col = u * 32 + lane;
      row_tok[u] = col < q_rows ? col / M.G : INT32_MAX;
      row_at[u] = col / M.G * M.Hq + col % M.G;
    }
    Ring kr, qr;
    uint32_t landed = 0;                  // parity of the next Q tile that the loader itself waits for
    bool k_used = false, q_used = false;  // the ring has been filled once: its slots have to be released first
    while (ok && walk.next(p, pl, sg)) {
      if (sg.n == 0) continue;
      const int32_t* tbl = p.b.block_table + (int64_t)sg.r * p.b.max_blocks;
      const int n_pages = (sg.kv_len + M.P - 1) / M.P;
      auto page_of = [&](int t) { return lane < ppt && t * ppt + lane < n_pages ? tbl[t * ppt + lane] : 0; };
      int pid_next = page_of(sg.t_lo);
      auto load_k = [&](int t) {
        if (t >= sg.t_hi || !ok) return;
        const int stage = kr.slot, pid = pid_next, pgi = t * ppt + lane;
        pid_next = page_of(t + 1);
        if (k_used && !warp_wait(bar(B_KEMPTY + stage), kr.phase ^ 1u)) {
          if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, sg.r, t, 90);
          ok = false;
          return;
        }
        bool mine = lane < ppt && pgi < n_pages;
        if (mine && (pid < 0 || pid >= p.num_pages)) {
          record_error(p.err, HSWA_ERR_BOUNDS, sg.r, pgi, pid);
          mine = false;
        }
        const int pages = __popc(__ballot_sync(0xffffffffu, mine));
        if (lane == 0) {
          if (pages == 0)
            mbar_arrive(bar(B_KFULL + stage));
          else
            mbar_arrive_expect_tx(bar(B_KFULL + stage), pages * M.P * 128 * HALVES);
        }
        __syncwarp();
        if (mine) {
          const uint32_t dst = sbase + off_k + stage * K_BYTES + lane * M.P * 128;
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf) tma_load_4d(dst + hf * K_HALF, &tm_pool, bar(B_KFULL + stage), hf * 64, 0, sg.kh, pid);
        }
        __syncwarp();
        kr.step(pl.nsk);
        k_used |= kr.slot == 0;
      };
      // lane's four rows of Q tile qt: minus their log-sum-exps in log2 units
      auto fetch_lse = [&](int qt, float(&x)[4]) {
        const float* lse = p.lse + (int64_t)(sg.t0 + qt * pl.tile_tokens) * M.Hq + sg.kh * M.G;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const float v = row_tok[u] < sg.n - qt * pl.tile_tokens ? lse[row_at[u]] : -INFINITY;
          x[u] = v == -INFINITY ? NO_ROW : -v * LOG2E;
        }
      };
      // The values of the next three Q tiles are on their way while one is staged (reading them one by one costs a memory
      // latency per Q tile).  fq: the next one to read, in the order in which the tiles are loaded.
      const int lo = first_qt(sg.t_lo);
      const bool resident = sg.n_qt - lo <= pl.nsq;
      float x[3][4];
      int fq = lo, ft = sg.t_lo;
      auto fetch_next = [&](float(&y)[4]) {
        if (fq < 0) return;
        fetch_lse(fq, y);
        if (++fq < sg.n_qt) return;
        ft += 2;
        fq = resident || ft >= sg.t_hi ? -1 : first_qt(ft);
      };
#pragma unroll
      for (int d = 0; d < 3; ++d) fetch_next(x[d]);
      auto load_q = [&](int qt) {
        const int stage = qr.slot;
        if (q_used && !warp_wait(bar(B_QEMPTY + stage), qr.phase ^ 1u)) {
          if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, sg.r, qt, 91);
          ok = false;
          return;
        }
        // A row whose lse is minus infinity adds nothing whatever its q holds, NaN included: it is zeroed between the tile's
        // arrival and its hand-over, so that its scores are finite.  (The loader waits for such tiles alone; dropping the row's
        // terms in the sums instead made every call 2 % slower.)
        bool drop[4], any = false;
#pragma unroll
        for (int u = 0; u < 4; ++u) any |= drop[u] = row_tok[u] < sg.n - qt * pl.tile_tokens && x[0][u] == NO_ROW;
        any = __any_sync(0xffffffffu, any);
        const uint32_t arrival = bar(any ? B_QLAND : B_QFULL + stage);
        if (lane == 0) {
          mbar_arrive_expect_tx(arrival, q_rows * 128 * HALVES);
#pragma unroll
          for (int hf = 0; hf < HALVES; ++hf)
            tma_load_3d(sbase + stage * q_bytes + hf * q_half, &tm_q, arrival, hf * 64, sg.kh * M.G, sg.t0 + qt * pl.tile_tokens);
        }
        if (any) {
          if (!warp_wait(arrival, landed)) {
            if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, sg.r, qt, 95);
            ok = false;
            return;
          }
          landed ^= 1u;
#pragma unroll
          for (int u = 0; u < 4; ++u)
            for (int i = 0; drop[u] && i < 8 * HALVES; ++i)
              *reinterpret_cast<uint4*>(smem + stage * q_bytes + (i >> 3) * q_half + (u * 32 + lane) * 128 + (i & 7) * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_QFULL + stage));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (u * 32 + lane < N) s_nl[stage * N + u * 32 + lane] = x[0][u];
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_LFULL + stage));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          x[0][u] = x[1][u];
          x[1][u] = x[2][u];
        }
        fetch_next(x[2]);
        qr.step(pl.nsq);
        q_used |= qr.slot == 0;
      };
      load_k(sg.t_lo);
      if (resident) {
        for (int qt = lo; qt < sg.n_qt && ok; ++qt) {
          load_q(qt);
          if (qt == lo) load_k(sg.t_lo + 1);
        }
        for (int t = sg.t_lo + 2; t < sg.t_hi && ok; ++t) load_k(t);
      } else {
        load_k(sg.t_lo + 1);
        for (int t = sg.t_lo; t < sg.t_hi && ok; t += 2) {
          const int first = first_qt(t);
          for (int qt = first; qt < sg.n_qt && ok; ++qt) {
            load_q(qt);
            if (qt == first) {  // the next pair of key tiles, behind this pair's first Q tile
              load_k(t + 2);
              load_k(t + 3);
            }
          }
        }
      }
    }
  } else if (warp == ISSUER) {
    // ======================= MMA issuer =======================
    const uint32_t idesc0 = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TKEYS >> 4) << 24);
    const uint64_t dQ0 = smem_desc(sbase, 16), dK0 = smem_desc(sbase + off_k, 16);
    bool ok = true;
    Ring kr, qr;
    int units[2] = {0, 0};
    while (ok && walk.next(p, pl, sg)) {
      if (sg.n == 0) continue;
      const int lo = first_qt(sg.t_lo);
      const bool resident = sg.n_qt - lo <= pl.nsq;
      for (int t = sg.t_lo; t < sg.t_hi && ok; t += 2) {
        const int first = first_qt(t);
        Ring k2 = kr, q = qr;  // the pair's second K tile; resident: the segment's Q tiles from its first one on
        k2.step(pl.nsk);
        if (resident) q.step(pl.nsq, first - lo);
        for (int qt = first; qt < sg.n_qt && ok; ++qt) {
          const int qs = q.slot;
          if (!resident || t == sg.t_lo) ok = warp_wait(bar(B_QFULL + qs), q.phase);
          // no more columns than the sums look at
          const int cols = min(pl.tile_tokens, sg.n - qt * pl.tile_tokens) * M.G;
          const uint32_t idesc = idesc0 | ((uint32_t)(mma_cols(cols, N) >> 3) << 17);
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (t + g >= sg.t_hi || !ok) continue;
            const int ks = g ? k2.slot : kr.slot, buf = units[g] & 1;
            if (qt == first) ok = warp_wait(bar(B_KFULL + ks), g ? k2.phase : kr.phase);
            if (ok && units[g] >= 2) ok = warp_wait(bar(B_SEMPTY + g * 2 + buf), ((units[g] >> 1) - 1) & 1);
            if (!ok) continue;
            tc_fence_after();
            if (elect_one()) {
              const uint64_t dk = desc_advance(dK0, ks * K_BYTES), dq = desc_advance(dQ0, qs * q_bytes);
#pragma unroll
              for (int s = 0; s < D / 16; ++s)
                tc_mma_ss(tmem + (g * 2 + buf) * N, desc_advance(dk, (s >> 2) * K_HALF + (s & 3) * 32),
                          desc_advance(dq, (s >> 2) * q_half + (s & 3) * 32), idesc, s > 0);
              tc_commit(bar(B_SFULL + g * 2 + buf));
              if (qt == sg.n_qt - 1) tc_commit(bar(B_KEMPTY + ks));
            }
            __syncwarp();
            ++units[g];
          }
          if (ok && !resident) {
            if (elect_one()) tc_commit(bar(B_QEMPTY + qs));
            __syncwarp();
          }
          q.step(pl.nsq);
        }
        if (!resident) qr = q;
        kr = k2;
        if (t + 1 < sg.t_hi) kr.step(pl.nsk);
      }
      if (ok && resident) {
        for (int qt = lo; qt < sg.n_qt; ++qt) {
          if (elect_one()) tc_commit(bar(B_QEMPTY + qr.slot));
          __syncwarp();
          qr.step(pl.nsq);
        }
      }
    }
    if (!ok && lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, sg.r, sg.kh, 92);
  } else {
    // ======================= sums =======================
    const int g = warp / GW, half = (warp % GW) >> 2, quad = warp & 3;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    bool ok = true;
    Ring qr;
    int units = 0;
    uint32_t joined = 0;  // bit b: parity of the next joining in accumulator b
    while (ok && walk.next(p, pl, sg)) {
      float* w_row = p.weights + ((int64_t)sg.r * M.Hkv + sg.kh) * p.stride;
      const int own = g * TKEYS + quad * 32 + lane;
      auto fetch_old = [&](int t) {  // positions of this step start at nothing
        const int j = t * TKEYS + own;
        return half == 0 && t + g < sg.t_hi && j < sg.ctx && p.decay != 0.f ? w_row[j] : 0.f;
      };
      float old_next = fetch_old(sg.t_lo);
      const int lo = first_qt(sg.t_lo);
      const bool resident = sg.n_qt - lo <= pl.nsq;
      for (int t = sg.t_lo; t < sg.t_hi && ok; t += 2) {
        const bool mine = t + g < sg.t_hi;
        const int j = t * TKEYS + own;
        const float old = old_next;
        old_next = fetch_old(t + 2);
        float sum = 0.f;
        const int first = first_qt(t);
        Ring q = qr;
        if (resident) q.step(pl.nsq, first - lo);
        for (int qt = first; qt < sg.n_qt && ok; ++qt) {
          const int qs = q.slot;
          if (!resident || t == sg.t_lo) ok = warp_wait(bar(B_LFULL + qs), q.phase);
          if (mine) {
            const int buf = units & 1;
            if (ok) ok = warp_wait(bar(B_SFULL + g * 2 + buf), (units >> 1) & 1);
            if (!ok) break;
            ++units;
            tc_fence_after();
            const uint32_t ts = tmem + lane_addr + (g * 2 + buf) * N;
            const float* nl = s_nl + qs * N;
            const int tok0 = qt * pl.tile_tokens;
            const int cols = min(pl.tile_tokens, sg.n - tok0) * M.G;
            const int full_cols = cols == q_rows ? mma_cols(cols, N) : cols;  // (a full tile's rows behind q_rows are zeros)
            // Columns [c_lo, cols) count: behind cols are rows of another request, before c_lo tokens that come before the
            // key.  Chunks that every lane of the warp sees whole take the short way, chunks that none sees are passed over.
            // (Clamped before it is multiplied: G times a far context passes 32 bits.)
            const int c_lo = p.causal ? max(0, j - sg.ctx - tok0) * M.G : 0;
            const int warp_lo = __shfl_sync(0xffffffffu, c_lo, 0), warp_hi = __shfl_sync(0xffffffffu, c_lo, 31);
            float2 acc[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
            const int c_begin = WIDE ? half * 64 : 0, c_end = WIDE ? min(cols, half * 64 + 64) : cols;
            if (WIDE && warp_hi <= c_begin && full_cols >= c_begin + 64) {
              // all 64 columns count: the next sixteen are read from TMEM while these are worked on
              uint32_t va[16], vb[16];
              tmem_ld16(ts + c_begin, va);
              tc_wait_ld();
              tmem_ld16(ts + c_begin + 16, vb);
              sum_chunk<false>(va, nl + c_begin, M.scale_log2, 0, 0, 0, acc);
              tc_wait_ld();
              tmem_ld16(ts + c_begin + 32, va);
              sum_chunk<false>(vb, nl + c_begin + 16, M.scale_log2, 0, 0, 0, acc);
              tc_wait_ld();
              tmem_ld16(ts + c_begin + 48, vb);
              sum_chunk<false>(va, nl + c_begin + 32, M.scale_log2, 0, 0, 0, acc);
              tc_wait_ld();
              sum_chunk<false>(vb, nl + c_begin + 48, M.scale_log2, 0, 0, 0, acc);
            } else {
#pragma unroll 1
              for (int c0 = max(warp_lo & ~15, c_begin); c0 < c_end; c0 += 16) {
                uint32_t v[16];
                tmem_ld16(ts + c0, v);
                tc_wait_ld();
                if (c0 >= warp_hi && c0 + 16 <= full_cols)
                  sum_chunk<false>(v, nl + c0, M.scale_log2, 0, 0, 0, acc);
                else
                  sum_chunk<true>(v, nl + c0, M.scale_log2, c0, c_lo, cols, acc);
              }
            }
            const float2 a = __fadd2_rn(__fadd2_rn(acc[0], acc[1]), __fadd2_rn(acc[2], acc[3]));
            sum += a.x + a.y;
            if (WIDE && qt == sg.n_qt - 1) {
              // The key's two sums meet: the upper columns' goes through the first of those columns, which its warps have
              // read by now.  The accumulator is free again when both halves have arrived below.
              if (half == 1) {
                tmem_st1(ts + 64, __float_as_uint(sum));
                tc_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_PFULL + g * 2 + buf));
              } else {
                ok = warp_wait(bar(B_PFULL + g * 2 + buf), (joined >> buf) & 1);
                joined ^= 1u << buf;
                if (!ok) break;
                tc_fence_after();
                uint32_t other;
                tmem_ld1(ts + 64, other);
                tc_wait_ld();
                sum += __uint_as_float(other);
              }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_SEMPTY + g * 2 + buf));
          }
          if (!resident) {
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(B_QEMPTY + qs));
          }
          q.step(pl.nsq);
        }
        if (!resident) qr = q;
        if (ok && half == 0 && mine && j < sg.kv_len) w_row[j] = p.decay != 0.f && j < sg.ctx ? fmaf(p.decay, old, sum) : sum;
      }
      if (ok && resident) {
        __syncwarp();
        for (int qt = lo; qt < sg.n_qt; ++qt) {
          if (lane == 0) mbar_arrive(bar(B_QEMPTY + qr.slot));
          qr.step(pl.nsq);
        }
      }
    }
    if (!ok && lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, sg.r, sg.kh, 93 + g);
  }
  // A role that gave up may leave TMA loads in flight towards this block's shared memory; outwait them.
  if (*reinterpret_cast<volatile int32_t*>(p.err) == HSWA_ERR_TIMEOUT) __nanosleep(100000);
  tc_fence_before();
  __syncthreads();
  if (warp == ISSUER) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(pl.tmem_cols) : "memory");
  }
}

template <int D, bool WIDE>
cudaError_t launch_t(const CUtensorMap& tm_pool, const CUtensorMap& tm_q, const WeightsParams& p, const WeightsPlan& pl, int blocks,
                     cudaStream_t s) {
  constexpr int HALVES = D / 64;
  int smem = pl.nsq * pl.n_cols * 128 * HALVES + pl.nsk * TKEYS * 128 * HALVES + pl.nsq * pl.n_cols * 4 + NUM_BARS * 8 + 32;
  if (WIDE && smem < 120 * 1024) smem = 120 * 1024;  // one block per SM: it takes all of its TMEM
  auto kern = attn_weights_kernel<D, WIDE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  kern<<<blocks, block_threads(WIDE), smem, s>>>(tm_pool, tm_q, p, pl);
  return cudaGetLastError();
}

}  // namespace

int hswa_attn_weights_tile_tokens(const ModelParams& m, int max_q_len) {
  const int most = 128 / m.G;
  return max_q_len < 1 ? 1 : (max_q_len < most ? max_q_len : most);
}

cudaError_t hswa_launch_attn_weights(const CUtensorMap& tm_pool, const CUtensorMap& tm_q, const WeightsParams& p, int num_sms,
                                     cudaStream_t s) {
  WeightsPlan pl = {};
  pl.tile_tokens = hswa_attn_weights_tile_tokens(p.m, p.max_q_len);
  const int rows = pl.tile_tokens * p.m.G;
  pl.n_cols = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 128;
  pl.tmem_cols = 4 * pl.n_cols;
  const int max_qt = (p.max_q_len + pl.tile_tokens - 1) / pl.tile_tokens;
  const bool wide = pl.n_cols > 64;
  const int tile_kb = p.m.D / 4;  // a tile of 128 rows
  if (wide) {
    // One block per SM, as many tiles as its shared memory holds: a Q stage more than a request has Q tiles (the next
    // segment's first one) as long as three K stages are left; where Q tiles are streamed, four K stages (the next pair's
    // are loaded while this one is multiplied) and the rest for Q
    const int stages = p.m.D == 128 ? 7 : 13;
    pl.nsq = max_qt + 1 < MAX_NSQ ? max_qt + 1 : MAX_NSQ;
    if (pl.nsq > stages - 3) pl.nsq = stages - 3;
    if (max_qt > pl.nsq && pl.nsq > stages - 4) pl.nsq = stages - 4;
    pl.nsk = stages - pl.nsq;
  } else {
    // two blocks per SM with 96 KB of K tiles each, beside one or two Q tiles of at most 16 KB
    pl.nsq = pl.n_cols == 64 && p.m.D == 128 ? 1 : 2;
    pl.nsk = 96 / tile_kb;
  }
  if (pl.nsk > MAX_NSK) pl.nsk = MAX_NSK;
  const int64_t keys = (int64_t)p.max_ctx_len + (p.causal ? p.max_q_len : 0);
  const int64_t tiles = (keys + TKEYS - 1) / TKEYS * p.m.Hkv * p.b.B, most = (wide ? 1 : 2) * (int64_t)num_sms;
  const int blocks = (int)(2 * tiles < most ? 2 * tiles : most);  // (a share ends between tiles: half of few blocks may be idle)
  if (p.m.D == 128) return wide ? launch_t<128, true>(tm_pool, tm_q, p, pl, blocks, s) : launch_t<128, false>(tm_pool, tm_q, p, pl, blocks, s);
  return wide ? launch_t<64, true>(tm_pool, tm_q, p, pl, blocks, s) : launch_t<64, false>(tm_pool, tm_q, p, pl, blocks, s);
}
