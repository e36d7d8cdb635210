// Accumulated attention weights of the cached keys (hswa_attn_weights): weights[j] = decay * weights[j] + the sum over the
// step's rows (token, head of the group) of exp(scale q.k_j - lse), for every (request, KV head).
//
// A score product whose output is summed over its ROWS: keys are the M dimension of tcgen05.mma (128 keys = 128 TMEM lanes
// = 128 threads), the packed (token, head) rows are N, so that a thread owns a key, adds up its row sums in registers and
// writes one number; nothing is exchanged between threads, no atomics, and the order of the sums is fixed.  Each key is
// read from memory once.
//
// Bounds.  One row group (a decode step) is bound by reading K.  With many rows the exponentials bound it: 16 per clock
// and SM against 32 score elements per clock from the tensor core at D = 128.
//
// Warp roles: warps 0-3 and 4-7 sum the even and the odd key tiles of the block's key range, warp 8 loads (TMA) and stages
// the rows' log-sum-exps, warp 9 issues the MMAs.  Each of the two summing groups has two TMEM accumulators.  The Q tiles
// (up to 128 rows) stay in shared memory for the block's whole key range when they all fit (up to 512 rows), else they are
// streamed from L2 once per pair of key tiles.
#include "hswa_internal.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int TKEYS = 128;       // keys per tile
constexpr int THREADS = 320;     // two summing groups, loader, MMA issuer
constexpr int MAX_NSQ = 4, MAX_NSK = 6;
constexpr float LOG2E = 1.4426950408889634f;

// Barriers
enum { B_QFULL = 0, B_LFULL = B_QFULL + MAX_NSQ, B_QEMPTY = B_LFULL + MAX_NSQ, B_KFULL = B_QEMPTY + MAX_NSQ,
       B_KEMPTY = B_KFULL + MAX_NSK, B_SFULL = B_KEMPTY + MAX_NSK /* [group][buffer] */, B_SEMPTY = B_SFULL + 4, NUM_BARS = B_SEMPTY + 4 };

struct WeightsPlan {
  int n_cols;       // N of the MMA: rows of a Q tile, rounded up
  int tile_tokens;  // tokens per Q tile
  int nsq, nsk;     // Q and K stages
  int resident;     // the Q tiles of a request all fit the Q stages
  int block_tiles;  // key tiles per block
  int tmem_cols;
};

// Index of the error word for a request that the host's bounds, the block table or the weights do not cover; 0 if fine.
__device__ __forceinline__ int weights_request_error(const WeightsParams& p, int ctx, int n) {
  if (ctx < 0 || ctx > p.max_ctx_len) return -1;
  if (n < 0 || n > p.max_q_len) return -2;
  const int64_t keys = (int64_t)ctx + (p.causal ? n : 0);
  return keys > p.stride || keys > (int64_t)p.b.max_blocks * p.m.P ? -3 : 0;
}

// A warp's bounded wait: one answer for all lanes.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }

// One thread's sum over CHUNK score columns.  nl: minus the rows' log-sum-exps in log2 units; a column that does not count
// (an absent row) has minus infinity there and a finite score.  MASKED: columns outside [c_lo, c_hi) are dropped whatever
// their score is.
template <int CHUNK, bool MASKED>
__device__ __forceinline__ void sum_chunk(const uint32_t (&v)[CHUNK], const float* nl, float scale_log2, int c0, int c_lo, int c_hi,
                                          float2 (&acc)[4]) {
  const float2 sc2 = make_float2(scale_log2, scale_log2);
#pragma unroll
  for (int k = 0; k < CHUNK; k += 4) {
    const float4 l4 = *reinterpret_cast<const float4*>(nl + k);
    const float2 x0 = __ffma2_rn(make_float2(__uint_as_float(v[k]), __uint_as_float(v[k + 1])), sc2, make_float2(l4.x, l4.y));
    const float2 x1 = __ffma2_rn(make_float2(__uint_as_float(v[k + 2]), __uint_as_float(v[k + 3])), sc2, make_float2(l4.z, l4.w));
    float2 e0 = make_float2(fast_exp2(x0.x), fast_exp2(x0.y)), e1 = make_float2(fast_exp2(x1.x), fast_exp2(x1.y));
    if constexpr (MASKED) {
      e0.x = c0 + k >= c_lo && c0 + k < c_hi ? e0.x : 0.f;
      e0.y = c0 + k + 1 >= c_lo && c0 + k + 1 < c_hi ? e0.y : 0.f;
      e1.x = c0 + k + 2 >= c_lo && c0 + k + 2 < c_hi ? e1.x : 0.f;
      e1.y = c0 + k + 3 >= c_lo && c0 + k + 3 < c_hi ? e1.y : 0.f;
    }
    acc[(k >> 1) & 3] = __fadd2_rn(acc[(k >> 1) & 3], e0);
    acc[((k >> 1) + 1) & 3] = __fadd2_rn(acc[((k >> 1) + 1) & 3], e1);
  }
}

// WIDE: one block per SM, Q tiles of up to 128 rows; else two blocks per SM (at most 64 rows), which hide each other's
// start and end.
template <int D, bool WIDE>
__global__ void __launch_bounds__(THREADS, WIDE ? 1 : 2)
attn_weights_kernel(const __grid_constant__ CUtensorMap tm_pool, const __grid_constant__ CUtensorMap tm_q, const WeightsParams p,
                    const WeightsPlan pl) {
  constexpr int HALVES = D / 64;
  constexpr int K_HALF = TKEYS * 128, K_BYTES = HALVES * K_HALF;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t sbase = smem_u32(smem);
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kh = blockIdx.y, r = blockIdx.z;
  const int N = pl.n_cols;
  const uint32_t q_half = (uint32_t)N * 128, q_bytes = q_half * HALVES;
  const uint32_t off_k = pl.nsq * q_bytes, off_lse = off_k + pl.nsk * K_BYTES;
  float* s_nl = reinterpret_cast<float*>(smem + off_lse);                            // [nsq][N]
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + off_lse + pl.nsq * N * 4);     // [NUM_BARS]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + NUM_BARS);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  const int t0 = p.b.q_indptr ? p.b.q_indptr[r] : r;
  const int n = p.b.q_indptr ? p.b.q_indptr[r + 1] - t0 : 1;
  const int ctx = p.b.ctx_len[r];
  const int bad = weights_request_error(p, ctx, n);
  if (bad != 0) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && kh == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, bad, bad == -1 ? ctx : bad == -2 ? n : ctx + n);
    return;
  }
  const int kv_len = ctx + (p.causal ? n : 0);
  const int k_begin = blockIdx.x * pl.block_tiles * TKEYS;
  if (k_begin >= kv_len) return;
  const int k_end = min(kv_len, k_begin + pl.block_tiles * TKEYS);
  const int n_tiles = (k_end - k_begin + TKEYS - 1) / TKEYS;
  const int n_qt = (n + pl.tile_tokens - 1) / pl.tile_tokens;
  float* w_row = p.weights + ((int64_t)r * M.Hkv + kh) * p.stride;
  if (n == 0) {  // no rows: the old weights only decay
    for (int j = k_begin + threadIdx.x; j < k_end; j += THREADS) w_row[j] = p.decay != 0.f ? p.decay * w_row[j] : 0.f;
    return;
  }
  // Q tiles that come before the first token which sees any key of tile t (causal: token i sees j <= ctx + i)
  auto first_qt = [&](int t) {
    const int over = k_begin + t * TKEYS - ctx;
    return p.causal && over > 0 ? over / pl.tile_tokens : 0;
  };

  if (threadIdx.x == 0) {
    for (int i = 0; i < pl.nsq; ++i) {
      mbar_init(bar(B_QFULL + i), 1);
      mbar_init(bar(B_LFULL + i), 1);
      mbar_init(bar(B_QEMPTY + i), 9);  // the MMA commit and eight summing warps
    }
    for (int i = 0; i < pl.nsk; ++i) {
      mbar_init(bar(B_KFULL + i), 1);
      mbar_init(bar(B_KEMPTY + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_SEMPTY + i), 4);
    }
    mbar_fence_init();
    if (sbase & 1023u) record_error(p.err, HSWA_ERR_CUDA, -1, (int)(sbase & 1023u), 16);  // tiles would be misread
  }
  // rows of a Q tile that no load fills (a group that does not divide 128): zeros, so that their scores are finite
  const int q_rows = pl.tile_tokens * M.G;
  for (int i = threadIdx.x; i < pl.nsq * HALVES * (N - q_rows) * 8; i += THREADS) {
    const int ch = i & 7, row = q_rows + (i >> 3) % (N - q_rows), hs = (i >> 3) / (N - q_rows);
    *reinterpret_cast<uint4*>(smem + (hs / HALVES) * q_bytes + (hs % HALVES) * q_half + row * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(pl.tmem_cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 8) {
    // ======================= loader =======================
    if (lane == 0) {
      tma_prefetch_desc(&tm_pool);
      tma_prefetch_desc(&tm_q);
    }
    const int n_pages = (k_end - k_begin + M.P - 1) / M.P, ppt = TKEYS / M.P;
    const int32_t* tbl = p.b.block_table + (int64_t)r * p.b.max_blocks + k_begin / M.P;
    int pid_next = lane < ppt && lane < n_pages ? tbl[lane] : 0;
    bool ok = true;
    auto load_k = [&](int t) {
      if (t >= n_tiles || !ok) return;
      const int stage = t % pl.nsk;
      const int pid = pid_next, pgi = t * ppt + lane;
      const int nx = pgi + ppt;
      pid_next = lane < ppt && nx < n_pages ? tbl[nx] : 0;
      if (t >= pl.nsk && !warp_wait(bar(B_KEMPTY + stage), ((t / pl.nsk) - 1) & 1)) {
        if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, t, 90);
        ok = false;
        return;
      }
      bool mine = lane < ppt && pgi < n_pages;
      if (mine && (pid < 0 || pid >= p.num_pages)) {
        record_error(p.err, HSWA_ERR_BOUNDS, r, k_begin / M.P + pgi, pid);
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
        for (int hf = 0; hf < HALVES; ++hf) tma_load_4d(dst + hf * K_HALF, &tm_pool, bar(B_KFULL + stage), hf * 64, 0, kh, pid);
      }
      __syncwarp();
    };
    // lane's four rows of Q tile qt: minus their log-sum-exps in log2 units (absent rows, and rows that saw nothing: minus
    // infinity, so that they add exp2(-inf) = 0)
    auto fetch_lse = [&](int qt, float (&x)[4]) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int col = u * 32 + lane, tok = qt * pl.tile_tokens + col / M.G;
        const float v = col < q_rows && tok < n ? p.lse[(int64_t)(t0 + tok) * M.Hq + kh * M.G + col % M.G] : -INFINITY;
        x[u] = v == -INFINITY ? -INFINITY : -v * LOG2E;
      }
    };
    auto load_q = [&](int qt, int stage, const float (&x)[4]) {
      if (lane == 0) {
        mbar_arrive_expect_tx(bar(B_QFULL + stage), q_rows * 128 * HALVES);
#pragma unroll
        for (int hf = 0; hf < HALVES; ++hf)
          tma_load_3d(sbase + stage * q_bytes + hf * q_half, &tm_q, bar(B_QFULL + stage), hf * 64, kh * M.G, t0 + qt * pl.tile_tokens);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (u * 32 + lane < N) s_nl[stage * N + u * 32 + lane] = x[u];
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_LFULL + stage));
    };
    float x[4];
    if (pl.resident) {
      load_k(0);
      for (int qt = 0; qt < n_qt; ++qt) {
        fetch_lse(qt, x);
        load_q(qt, qt, x);
        if (qt == 0) load_k(1);
      }
      for (int t = 2; t < n_tiles && ok; ++t) load_k(t);
    } else {
      load_k(0);
      load_k(1);
      int qi = 0;
      fetch_lse(first_qt(0), x);
      for (int t = 0; t < n_tiles && ok; t += 2) {
        const int lo = first_qt(t);
        for (int qt = lo; qt < n_qt && ok; ++qt, ++qi) {
          const int stage = qi % pl.nsq;
          if (qi >= pl.nsq && !warp_wait(bar(B_QEMPTY + stage), ((qi / pl.nsq) - 1) & 1)) {
            if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, qi, 91);
            ok = false;
            break;
          }
          load_q(qt, stage, x);
          fetch_lse(qt + 1 < n_qt ? qt + 1 : first_qt(t + 2), x);  // the next one's values are under way meanwhile
          if (qt == lo) {  // the next pair of key tiles, behind this pair's first Q tile
            load_k(t + 2);
            load_k(t + 3);
          }
        }
      }
    }
  } else if (warp == 9) {
    // ======================= MMA issuer =======================
    const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(TKEYS >> 4) << 24);
    const uint64_t dQ0 = smem_desc(sbase, 16), dK0 = smem_desc(sbase + off_k, 16);
    bool ok = true;
    int qi = 0, units[2] = {0, 0};
    for (int t = 0; t < n_tiles && ok; t += 2) {
      const int lo = first_qt(t);
      for (int qt = lo; qt < n_qt && ok; ++qt, ++qi) {
        const int qs = pl.resident ? qt : qi % pl.nsq;
        ok = warp_wait(bar(B_QFULL + qs), pl.resident ? 0 : (qi / pl.nsq) & 1);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (t + g >= n_tiles || !ok) continue;
          const int ks = (t + g) % pl.nsk, buf = units[g] & 1;
          if (qt == lo) ok = warp_wait(bar(B_KFULL + ks), ((t + g) / pl.nsk) & 1);
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
            if (qt == n_qt - 1) tc_commit(bar(B_KEMPTY + ks));
          }
          __syncwarp();
          ++units[g];
        }
        if (ok && !pl.resident) {
          if (elect_one()) tc_commit(bar(B_QEMPTY + qs));
          __syncwarp();
        }
      }
    }
    if (!ok && lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, qi, 92);
  } else {
    // ======================= sums =======================
    const int g = warp >> 2, quad = warp & 3;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    bool ok = true;
    int qi = 0, units = 0;
    uint32_t seen_l = 0;  // resident: bit qt = the tile's log-sum-exps have been waited for
    float old_next = 0.f;
    auto fetch_old = [&](int t) {
      const int j = k_begin + t * TKEYS + quad * 32 + lane;
      return t < n_tiles && j < k_end && j < ctx && p.decay != 0.f ? w_row[j] : 0.f;
    };
    old_next = fetch_old(g);
    for (int t = 0; t < n_tiles && ok; t += 2) {
      const bool mine = t + g < n_tiles;
      const int j = k_begin + (t + g) * TKEYS + quad * 32 + lane;
      const float old = old_next;
      old_next = fetch_old(t + 2 + g);
      const int last_key = k_begin + (t + g) * TKEYS + TKEYS - 1;
      float sum = 0.f;
      for (int qt = first_qt(t); qt < n_qt && ok; ++qt, ++qi) {
        const int qs = pl.resident ? qt : qi % pl.nsq;
        if (!pl.resident) {
          ok = warp_wait(bar(B_LFULL + qs), (qi / pl.nsq) & 1);
        } else if (!((seen_l >> qt) & 1u)) {
          ok = warp_wait(bar(B_LFULL + qs), 0);
          seen_l |= 1u << qt;
        }
        if (mine) {
          const int buf = units & 1;
          if (ok) ok = warp_wait(bar(B_SFULL + g * 2 + buf), (units >> 1) & 1);
          if (!ok) break;
          ++units;
          tc_fence_after();
          const uint32_t ts = tmem + lane_addr + (g * 2 + buf) * N;
          const float* nl = s_nl + qs * N;
          const int tok0 = qt * pl.tile_tokens;
          const int cols = min(pl.tile_tokens, n - tok0) * M.G;
          // rows of another request behind this one's last token, or keys ahead of some of the tile's tokens
          const bool masked = cols < q_rows || (p.causal && last_key > ctx + tok0);
          const int c_lo = p.causal ? (j - ctx - tok0) * M.G : 0;
          float2 acc[4];
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
          if (N == 16) {
            uint32_t v[16];
            tmem_ld16(ts, v);
            tc_wait_ld();
            if (masked) sum_chunk<16, true>(v, nl, M.scale_log2, 0, c_lo, cols, acc);
            else sum_chunk<16, false>(v, nl, M.scale_log2, 0, c_lo, cols, acc);
          } else if (masked) {
            for (int c0 = 0; c0 < N; c0 += 32) {
              uint32_t v[32];
              tmem_ld32(ts + c0, v);
              tc_wait_ld();
              sum_chunk<32, true>(v, nl + c0, M.scale_log2, c0, c_lo, cols, acc);
            }
          } else {
            for (int c0 = 0; c0 < N; c0 += 32) {
              uint32_t v[32];
              tmem_ld32(ts + c0, v);
              tc_wait_ld();
              sum_chunk<32, false>(v, nl + c0, M.scale_log2, c0, c_lo, cols, acc);
            }
          }
          const float2 a = __fadd2_rn(__fadd2_rn(acc[0], acc[1]), __fadd2_rn(acc[2], acc[3]));
          sum += a.x + a.y;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_SEMPTY + g * 2 + buf));
        }
        if (!pl.resident) {
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(B_QEMPTY + qs));
        }
      }
      if (ok && mine && j < k_end) w_row[j] = p.decay != 0.f && j < ctx ? fmaf(p.decay, old, sum) : sum;
    }
    if (!ok && lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, qi, 93 + g);
  }
  // A role that gave up may leave TMA loads in flight towards this block's shared memory; outwait them.
  if (*reinterpret_cast<volatile int32_t*>(p.err) == HSWA_ERR_TIMEOUT) __nanosleep(100000);
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(pl.tmem_cols) : "memory");
  }
}

template <int D, bool WIDE>
cudaError_t launch_t(const CUtensorMap& tm_pool, const CUtensorMap& tm_q, const WeightsParams& p, const WeightsPlan& pl, cudaStream_t s) {
  constexpr int HALVES = D / 64;
  int smem = pl.nsq * pl.n_cols * 128 * HALVES + pl.nsk * TKEYS * 128 * HALVES + pl.nsq * pl.n_cols * 4 + NUM_BARS * 8 + 16;
  if (WIDE && smem < 120 * 1024) smem = 120 * 1024;  // one block per SM: it takes all of its TMEM
  auto kern = attn_weights_kernel<D, WIDE>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int64_t keys = (int64_t)p.max_ctx_len + (p.causal ? p.max_q_len : 0);
  const int64_t tiles = (keys + TKEYS - 1) / TKEYS;
  dim3 grid((unsigned)((tiles + pl.block_tiles - 1) / pl.block_tiles), p.m.Hkv, p.b.B);
  kern<<<grid, THREADS, smem, s>>>(tm_pool, tm_q, p, pl);
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
  pl.resident = max_qt <= MAX_NSQ;
  pl.nsq = max_qt < 1 ? 1 : (pl.resident ? max_qt : 3);
  const int tile_kb = p.m.D / 4;  // a 128-row tile
  // shared memory: 224 KB of tiles in one block per SM, 96 KB of K tiles beside one small Q tile in each of two
  pl.nsk = wide ? (224 - pl.nsq * tile_kb) / tile_kb : 96 / tile_kb;
  if (pl.nsk > MAX_NSK) pl.nsk = MAX_NSK;
  // Key tiles per block: long enough to pay for a block's start, short enough to fill the machine
  const int64_t keys = (int64_t)p.max_ctx_len + (p.causal ? p.max_q_len : 0);
  const int64_t tiles = (keys + TKEYS - 1) / TKEYS;
  int per = 32;
  while (per > 2 && (int64_t)p.b.B * p.m.Hkv * ((tiles + per - 1) / per) < 4LL * num_sms) per >>= 1;
  pl.block_tiles = per;
  if (p.m.D == 128) return wide ? launch_t<128, true>(tm_pool, tm_q, p, pl, s) : launch_t<128, false>(tm_pool, tm_q, p, pl, s);
  return wide ? launch_t<64, true>(tm_pool, tm_q, p, pl, s) : launch_t<64, false>(tm_pool, tm_q, p, pl, s);
}
