// Attention over a 4-bit cache for many rows per KV head (prompts) on the 5th-generation tensor cores: hswa_packed_attn.
//
// A block takes two Q tiles of 128 rows (128 / G tokens x the G query heads of one KV head) against one slice of the request's
// keys.  Warp roles:
//   warps 0-7    softmax, four per Q tile: TMEM lane = row = thread, which holds the 128 scores of its row; before the loop each
//                thread brings its row of Q into shared memory as fp16
//   warps 8, 9   MMA issuers, one per Q tile: S_i = Q_i K^T from shared memory, O_i += P_i V with P_i from TMEM, in turns, so that one
//                tile's softmax overlaps the other's MMAs
//   warps 12-15  unpackers: codes and scales of a 128-key tile from global memory to fp16 rows in swizzled shared memory, K and V in
//                rings of two tiles.  A lane holds 32 elements at a time; while it converts them, the same lane's next 32 are
//                on their way, so the latency of a load is that of half a tile's conversion.
// TMEM columns: S0 0-127, S1 128-255, O0 256-, O1 384- (fp32; P_i = fp16 pairs over the first 64 columns of S_i).  O is rescaled
// only when a row's base moves (packed.cuh).  Rows of a key tile that no row sees are written as zeros.
// Bound by the tensor cores and the exponentials; the unpackers' conversion (a fifth of the issue slots) hides beside them.  Measured, 8
// prompts of 257 to 512 tokens over up to 8192 keys, 64 / 8 heads of 128: 668 us alone, 1.03 PFLOP/s, 705 in a sustained run under the
// power cap (410 at the rate of a plain matrix product; blocks of warp-level MMAs took 5483).
#include "block_order.cuh"
#include "packed.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int BM = 128, BN = 128;
constexpr int HALF_BYTES = 128 * 128;  // [128 rows][128 B]: 64 elements of each row
constexpr int TILE_BYTES = 2 * HALF_BYTES;
constexpr int STAGES = 2;
constexpr int kThreads = 512;
constexpr int W_MMA = 8, W_UNPACK = 12;
// Registers per thread once the roles have split: their sum is what the launch gave (512 x 128).
constexpr int REGS_SOFTMAX = 200, REGS_MMA = 48, REGS_UNPACK = 64;
static_assert(2 * REGS_SOFTMAX + REGS_MMA + REGS_UNPACK == 4 * 128, "what the launch gave");

constexpr int OFF_Q = 0, OFF_K = 2 * TILE_BYTES, OFF_V = OFF_K + STAGES * TILE_BYTES, OFF_STATE = OFF_V + STAGES * TILE_BYTES;
constexpr int kSmem = OFF_STATE + 256;
constexpr int TM_O = 256, TM_COLS = 512;
constexpr int P_PARTS = 2;  // P goes to the MMA issuer in two halves of 64 keys

enum { BAR_Q = 0, BAR_KFULL = 1, BAR_KEMPTY = 3, BAR_VFULL = 5, BAR_VEMPTY = 7, BAR_SFULL = 9, BAR_PFULL = 11 /* [Q tile][half] */,
       BAR_OFINAL = 15 /* [Q tile] */, NUM_BARS = 17 };

// fp16 operands, fp32 accumulators
constexpr uint32_t IDESC_S = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);

template <int D>
__global__ void __launch_bounds__(kThreads, 1) packed_tile_kernel(const PackedAttnParams p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  constexpr uint32_t IDESC_O = (IDESC_S & ~(0x3fu << 17)) | ((uint32_t)(D >> 3) << 17) | (1u << 16);  // B (= V) is [key][d], d contiguous
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + OFF_STATE);
  uint32_t& tmem_base_slot = *reinterpret_cast<uint32_t*>(smem + OFF_STATE + 160);
  int& failed = *reinterpret_cast<int*>(smem + OFF_STATE + 164);
  int* picked = reinterpret_cast<int*>(smem + OFF_STATE + 168);
  int* issuer_stop = reinterpret_cast<int*>(smem + OFF_STATE + 176);  // [2] an MMA issuer is to stop: a wait ran out
  const uint32_t sbase = smem_u32(smem);
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // blockIdx.x = slice + slices * (KV head + Hkv * number of the row tile)
  const int slice = blockIdx.x % p.slices, kh = blockIdx.x / p.slices % M.Hkv, number = blockIdx.x / p.slices / M.Hkv;
  const int tok_tile = BM / M.G;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  // the grid was sized from the host's bounds
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < p.b.B; i += kThreads) {
      const int c = p.b.ctx_len[i], a = p.b.q_indptr[i], k = p.b.q_indptr[i + 1] - a;
      if (c < 0 || c > p.max_ctx_len) record_error(p.err, HSWA_ERR_BOUNDS, i, -1, c);
      if (k < 0 || k > p.max_q_len || a < 0 || (int64_t)a + k > p.total_q) record_error(p.err, HSWA_ERR_BOUNDS, i, -2, k);
      const int64_t sees = (int64_t)max(0, min(c, p.max_ctx_len)) + min(k, p.max_q_len);
      if (p.causal && k > 0 && sees > (int64_t)p.b.max_blocks * M.P) record_error(p.err, HSWA_ERR_BOUNDS, i, -3, (int)sees);
    }
  // longest request first, and its longest row tile first
  if (warp == 0) {
    int pr = -1, pb = 0;
    auto tiles_of = [&](int rq, int& key, int& nt) {
      nt = (min(p.b.q_indptr[rq + 1] - p.b.q_indptr[rq], p.max_q_len) + 2 * tok_tile - 1) / (2 * tok_tile);
      nt = max(nt, 0);
      key = nt > 0 ? 1 + max(0, min(p.b.ctx_len[rq], p.max_ctx_len)) / BN : 0;
    };
    if (!pick_longest_request_first(p.b, number, lane, tiles_of, &pr, &pb)) pr = -1;
    if (lane == 0) {
      picked[0] = pr;
      picked[1] = pb;
      issuer_stop[0] = issuer_stop[1] = 0;
      // an earlier block gave up: do not queue behind it
      failed = *reinterpret_cast<volatile int32_t*>(p.err) == HSWA_ERR_TIMEOUT;
      if (sbase & 1023u) {  // the swizzled tiles need a 1 KB-aligned window
        record_error(p.err, HSWA_ERR_CUDA, -1, (int)(sbase & 1023u), 15);
        failed = 1;
      }
    }
  }
  __syncthreads();
  const int r = picked[0], b = picked[1];
  if (r < 0 || failed) return;  // uniform for the block
  const int t0 = p.b.q_indptr[r], n_all = p.b.q_indptr[r + 1] - t0, n = min(n_all, p.max_q_len);
  auto has_row = [&](int tok) { return (unsigned)t0 + (unsigned)tok < (unsigned)p.total_q; };
  const int tok0 = b * 2 * tok_tile, tok_end = min(n, tok0 + 2 * tok_tile);
  const int len = max(0, min(p.b.ctx_len[r], p.max_ctx_len));
  const int64_t room = (int64_t)p.b.max_blocks * M.P;
  const int k0 = slice * p.slice_len;
  // keys of this slice that the block's last row sees
  const int keys = (int)min(min(room, (int64_t)(p.causal ? len + tok_end : len)) - k0, (int64_t)p.slice_len);
  const int n_tiles = keys > 0 ? (keys + BN - 1) / BN : 0;
  const int q_tiles = tok0 + tok_tile < n ? 2 : 1;

  if (p.slices > 1 && b == 0 && slice == 0) {
    // rows past the host's bound have no block: a mark tells the join to leave them alone
    for (int64_t tok = (int64_t)p.max_q_len + threadIdx.x; tok < n_all; tok += kThreads)
      if (has_row((int)tok))
        for (int g = 0; g < M.G; ++g) p.part_ml[(((int64_t)t0 + tok) * M.Hq + kh * M.G + g) * p.slices] = make_float2(-INFINITY, -1.f);
  }
  if (n_tiles == 0) {
    // no key here: zeros, or a partial that the join passes over
    for (int row = threadIdx.x; row < (tok_end - tok0) * M.G; row += kThreads) {
      const int tok = tok0 + row / M.G;
      if (!has_row(tok)) continue;
      const int64_t orow = (int64_t)(t0 + tok) * M.Hq + kh * M.G + row % M.G;
      if (p.slices > 1) {
        p.part_ml[orow * p.slices + slice] = make_float2(-INFINITY, 0.f);
        continue;
      }
      uint4* dst = M.out_fp32 ? reinterpret_cast<uint4*>(reinterpret_cast<float*>(p.out) + orow * D)
                              : reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D);
      for (int k = 0; k < (M.out_fp32 ? D / 4 : D / 8); ++k) dst[k] = make_uint4(0, 0, 0, 0);
      if (p.lse) p.lse[orow] = -INFINITY;
    }
    return;
  }

  if (threadIdx.x == 0) {
    mbar_init(bar(BAR_Q), 4 * q_tiles);  // one arrival per softmax warp
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(bar(BAR_KFULL + s), 4);  // one per unpacking warp
      mbar_init(bar(BAR_VFULL + s), 4);
      mbar_init(bar(BAR_KEMPTY + s), q_tiles);  // one commit per MMA issuer
      mbar_init(bar(BAR_VEMPTY + s), q_tiles);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(BAR_SFULL + i), 1);
      for (int q = 0; q < P_PARTS; ++q) mbar_init(bar(BAR_PFULL + P_PARTS * i + q), 4);
      mbar_init(bar(BAR_OFINAL + i), 1);
    }
    mbar_fence_init();
  }
  if (warp == W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_slot)), "r"(TM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_base_slot;

  if (warp >= W_UNPACK) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_UNPACK) : "memory");
    // ======================= unpackers =======================
    // A lane takes 16 bytes (32 elements, two scales) of `LOADS` rows of a tile.  Eight neighbouring lanes are on four rows and
    // two parts of a row: 32-byte sectors are read whole, and their 16-byte stores fall on eight different bank groups.
    constexpr int ROW = D / 2, SC = D / 16, LOADS = D / 32, STEP = BN / LOADS;
    const int u = warp - W_UNPACK;
    const int part = D == 128 ? (lane & 1) | ((lane >> 3) & 1) << 1 : lane & 1;
    const int row0 = D == 128 ? ((lane >> 1) & 3) | (lane >> 4) << 2 | u << 3 : ((lane >> 1) & 3) | (lane >> 3) << 2 | u << 4;
    const int slab = M.P * (ROW + SC), page_shift = 31 - __clz(M.P);
    const int32_t* tbl = p.b.block_table + (int64_t)r * p.b.max_blocks + (k0 >> page_shift);
    int pid[LOADS], pid_next[LOADS];  // page of each of the lane's rows: of the tile whose loads come next, and of the one behind
    uint4 data[LOADS];
    uint32_t f[LOADS];
    auto next_pages = [&](int j) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int key = j * BN + row0 + i * STEP;
        pid_next[i] = key < keys ? tbl[key >> page_shift] : 0;
      }
    };
    auto take_pages = [&](int j) {  // next_pages' of tile j
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int key = j * BN + row0 + i * STEP;
        pid[i] = key < keys ? pid_next[i] : -1;
        if (key < keys && (pid[i] < 0 || pid[i] >= p.num_pages)) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, (k0 + key) >> page_shift, pid[i]);
          pid[i] = 0;
        }
      }
    };
    auto load = [&](int i, int kv) {
      data[i] = make_uint4(0, 0, 0, 0);
      f[i] = 0;
      if (pid[i] >= 0) {
        const int slot = (row0 + i * STEP) & (M.P - 1);
        const uint8_t* at = p.pool + (((int64_t)pid[i] * 2 + kv) * M.Hkv + kh) * slab;
        data[i] = __ldg(reinterpret_cast<const uint4*>(at + slot * ROW + part * 16));
        f[i] = __ldg(reinterpret_cast<const uint16_t*>(at + M.P * ROW + slot * SC + part * 2));
      }
    };
    auto store = [&](int i, uint8_t* tile) {
      const uint32_t w[4] = {data[i].x, data[i].y, data[i].z, data[i].w};
      const uint32_t f2 = e4m3_to_half2(f[i]), s[2] = {low_twice(f2), high_twice(f2)};
      const int row = row0 + i * STEP;
      uint8_t* at = tile + (part >> 1) * HALF_BYTES;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t h = s[q >> 1];
        *reinterpret_cast<uint4*>(at + swz128(row, (part & 1) * 4 + q)) =
            make_uint4(hmul2(e2m1_to_half2<0>(w[q]), h), hmul2(e2m1_to_half2<1>(w[q]), h), hmul2(e2m1_to_half2<2>(w[q]), h),
                       hmul2(e2m1_to_half2<3>(w[q]), h));
      }
    };
    next_pages(0);
    take_pages(0);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) load(i, 0);
    bool ok = true;
    for (int j = 0; j < n_tiles && ok; ++j) {
      const int stage = j % STAGES;
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        if (j >= STAGES && !__all_sync(0xffffffffu, mbar_wait(bar((kv ? BAR_VEMPTY : BAR_KEMPTY) + stage), ((j / STAGES) - 1) & 1))) {
          if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 60 + kv);
          ok = false;
          break;
        }
        uint8_t* tile = smem + (kv ? OFF_V : OFF_K) + stage * TILE_BYTES;
        if (kv) take_pages(j + 1);  // (V of this tile is on its way)
        else next_pages(j + 1);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          store(i, tile);
          load(i, kv ^ 1);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar((kv ? BAR_VFULL : BAR_KFULL) + stage));
      }
    }
  } else if (warp >= W_MMA) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(REGS_MMA) : "memory");
    // ======================= MMA issuers =======================
    if (warp - W_MMA < q_tiles) {
      const int i = warp - W_MMA;
      // A wait may run out for some lanes of the warp alone, so none leaves by itself: it sets its warp's flag, and the warp leaves
      // behind the next barrier, where all lanes read the same.  The other issuer's flag is set with the token in hand.  (Votes on
      // the waits: 697 us against 672.)
      volatile int *stop = &issuer_stop[i], *stop_other = &issuer_stop[1 - i];
      auto await = [&](int which, uint32_t parity) {
        if (mbar_wait(bar(which), parity)) return true;
        record_error(p.err, HSWA_ERR_TIMEOUT, r, b, 62 + i);
        *stop = 1;
        return false;  // (of use to leave out waits behind it)
      };
      const bool q_here = await(BAR_Q, 0);
      const uint64_t dQ = smem_desc(sbase + OFF_Q + i * TILE_BYTES, 16);
      const uint64_t dK0 = smem_desc(sbase + OFF_K, 16), dV0 = smem_desc(sbase + OFF_V, HALF_BYTES);
      auto issue_S = [&](int stage) {
        tc_fence_after();
        const uint64_t dk = desc_advance(dK0, stage * TILE_BYTES);
        if (elect_one()) {
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks) {
            const uint32_t off = (ks >> 2) * HALF_BYTES + (ks & 3) * 32;
            tc_mma_ss(tmem + i * 128, desc_advance(dQ, off), desc_advance(dk, off), IDESC_S, ks > 0);
          }
          tc_commit(bar(BAR_SFULL + i));
          tc_commit(bar(BAR_KEMPTY + stage));
        }
        __syncwarp();
      };
      constexpr int KSTEPS = 8 / P_PARTS;
      auto issue_PV = [&](int stage, int part, bool first) {
        tc_fence_after();
        const uint64_t dv = desc_advance(dV0, stage * TILE_BYTES + part * KSTEPS * 2048);
        if (elect_one()) {
#pragma unroll
          for (int q = 0; q < KSTEPS; ++q)
            tc_mma_ts(tmem + TM_O + i * 128, tmem + i * 128 + (part * KSTEPS + q) * 8, desc_advance(dv, q * 2048), IDESC_O,
                      !(first && part == 0 && q == 0));
        }
        __syncwarp();
      };
      // [PV0(j), S0(j+1)] [PV1(j), S1(j+1)] ...: a token goes around through two named barriers.  An issuer leaves the loop only
      // right after passing the token, and passes it when it finds its flag set, so neither waits forever.  (A wait that runs
      // out with the token in hand is found at the next turn; the products until then are of a call that has failed.)
      const int tok_in = i == 0 ? 2 : 1, tok_out = i == 0 ? 1 : 2;
      auto token_wait = [&]() {
        if (q_tiles == 2) asm volatile("bar.sync %0, 64;" ::"r"(tok_in) : "memory");
        else __syncwarp();
      };
      auto token_pass = [&]() {
        if (q_tiles == 1) return;
        __threadfence_block();
        asm volatile("bar.arrive %0, 64;" ::"r"(tok_out) : "memory");
      };
      if (q_here) await(BAR_KFULL + 0, 0);
      if (i == 1) token_wait();
      else __syncwarp();
      if (*stop != 0) *stop_other = 1;
      else issue_S(0);
      token_pass();
      for (int j = 0; j < n_tiles; ++j) {
        const int stage = j % STAGES, nstage = (j + 1) % STAGES;
        const bool more = j + 1 < n_tiles;
        // polled during the other issuer's turn
        if (await(BAR_VFULL + stage, (j / STAGES) & 1) && await(BAR_PFULL + P_PARTS * i, j & 1) && more) await(BAR_KFULL + nstage, ((j + 1) / STAGES) & 1);
        token_wait();
        if (*stop != 0) {
          *stop_other = 1;
          token_pass();
          break;
        }
#pragma unroll
        for (int q = 0; q < P_PARTS; ++q) {
          if (q > 0) await(BAR_PFULL + P_PARTS * i + q, j & 1);
          issue_PV(stage, q, j == 0);
        }
        if (elect_one()) tc_commit(bar(BAR_VEMPTY + stage));
        __syncwarp();
        if (more) issue_S(nstage);
        token_pass();
      }
      if (elect_one()) tc_commit(bar(BAR_OFINAL + i));
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(REGS_SOFTMAX) : "memory");
    // ======================= softmax =======================
    const int i = warp >> 2, quad = warp & 3;
    const int rr = quad * 32 + lane;  // row of the Q tile = TMEM lane
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t tS = tmem + lane_addr + i * 128, tO = tmem + lane_addr + TM_O + i * 128;
    const int tok = tok0 + i * tok_tile + rr / M.G;
    const bool row_here = rr < tok_tile * M.G && tok < n && has_row(tok);
    const int64_t orow = (int64_t)(t0 + tok) * M.Hq + kh * M.G + rr % M.G;
    // keys of the slice that the row sees
    const int64_t sees64 = min(room, (int64_t)(p.causal ? len + tok + 1 : len)) - k0;
    const int sees = (int)max((int64_t)0, min(sees64, (int64_t)p.slice_len));
    float mul = 0.f;
    if (i < q_tiles) {
      const uint4* src = reinterpret_cast<const uint4*>(p.q + orow * D);
      float amax = 0.f;
#pragma unroll 4
      for (int k = 0; k < D / 8; ++k) {
        const uint4 v = row_here ? src[k] : make_uint4(0, 0, 0, 0);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = unpack_bf16x2(u[e]);
          amax = finite_max(amax, x);
        }
      }
      float up, down;
      q_powers(amax, &up, &down);
      mul = fmaxf(down * p.scale_log2, 0x1p-126f);  // (never 0: a masked score stays minus infinity)
#pragma unroll 4
      for (int k = 0; k < D / 8; ++k) {
        const uint4 v = row_here ? src[k] : make_uint4(0, 0, 0, 0);
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        uint32_t o[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = unpack_bf16x2(u[e]);
          o[e] = pack_half2(x.x * up, x.y * up);
        }
        *reinterpret_cast<uint4*>(smem + OFF_Q + i * TILE_BYTES + (k >> 3) * HALF_BYTES + swz128(rr, k & 7)) = make_uint4(o[0], o[1], o[2], o[3]);
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_Q));
    }
    float m_st = -INFINITY, l_run = 0.f;
    bool ok = true;
    for (int j = 0; j < (i < q_tiles ? n_tiles : 0); ++j) {
      ok = __all_sync(0xffffffffu, mbar_wait(bar(BAR_SFULL + i), j & 1));  // warp-uniform: TMEM operations are warp-wide
      if (!ok) {
        if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 64 + i);
        break;
      }
      const int hi = sees - j * BN;  // the row's first masked column
      uint32_t v[128];
      tc_fence_after();
      tmem_ld32(tS, v);
      tmem_ld32(tS + 32, v + 32);
      tmem_ld32(tS + 64, v + 64);
      tmem_ld32(tS + 96, v + 96);
      tc_wait_ld();
      if (__any_sync(0xffffffffu, hi < BN)) {
#pragma unroll
        for (int k = 0; k < 128; ++k)
          if (k >= hi) v[k] = 0xff800000u;  // -inf
      }
      float mx8[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) mx8[c] = fmaxf(__uint_as_float(v[2 * c]), __uint_as_float(v[2 * c + 1]));
#pragma unroll
      for (int k = 16; k < 128; k += 16) {
#pragma unroll
        for (int c = 0; c < 8; ++c) mx8[c] = max3(mx8[c], __uint_as_float(v[k + 2 * c]), __uint_as_float(v[k + 2 * c + 1]));
      }
      const float mx = fmaxf(fmaxf(max3(mx8[0], mx8[1], mx8[2]), max3(mx8[3], mx8[4], mx8[5])), fmaxf(mx8[6], mx8[7]));
      const float mx_s = base_of(mx, mul);
      if (j == 0) {
        m_st = mx_s;
      } else {
        const bool grow = base_moves(mx_s, m_st);
        if (__any_sync(0xffffffffu, grow)) {
          const float m_new = grow ? mx_s : m_st;
          const float alpha = (m_new == -INFINITY) ? 1.f : fast_exp2(m_st - m_new);
#pragma unroll 1
          for (int c16 = 0; c16 < D / 16; ++c16) {
            uint32_t w[16];
            tmem_ld16(tO + c16 * 16, w);
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(__uint_as_float(w[k]) * alpha);
            tmem_st16p(tO + c16 * 16, w);
          }
          l_run *= alpha;
          m_st = m_new;
        }
      }
      const float m_use = (m_st == -INFINITY) ? 0.f : m_st;
      const float2 sc2 = make_float2(mul, mul), nm2 = make_float2(-m_use, -m_use);
      float2 acc[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = make_float2(0.f, 0.f);
      constexpr int QPP = 4 / P_PARTS;  // 32-key quarters per posted part
#pragma unroll
      for (int part = 0; part < 4; ++part) {
#pragma unroll
        for (int k = part * 16; k < part * 16 + 16; ++k) {
          const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), sc2, nm2);
          const float2 e = make_float2(fast_exp2(x.x), fast_exp2(x.y));
          v[k] = pack_half2(e.x, e.y);
          acc[k & 3] = __fadd2_rn(acc[k & 3], e);  // (the row sum takes the values before their rounding to fp16)
          if (part > 0 && (part % QPP) == 0 && k == part * 16 + 7) {
            // post the previous half: its TMEM stores have landed by now
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(BAR_PFULL + P_PARTS * i + part / QPP - 1));
          }
        }
        tmem_st16p(tS + part * 16, v + part * 16);
        if (part == 3) {
          tc_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(BAR_PFULL + P_PARTS * i + P_PARTS - 1));
        }
      }
      const float2 a01 = __fadd2_rn(acc[0], acc[1]), a23 = __fadd2_rn(acc[2], acc[3]);
      l_run += (a01.x + a01.y) + (a23.x + a23.y);
    }
    // ---- O / l, or the slice's partial ----
    if (i < q_tiles) {
      if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(BAR_OFINAL + i), 0));
      if (!ok && lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, b, 66 + i);
      tc_fence_after();
      const bool some = l_run != 0.f;  // (a NaN among the inputs shows in the output)
      const float inv = p.slices > 1 ? p.v_scale : (some ? p.v_scale / l_run : 0.f);
      const bool to_fp32 = p.slices > 1 || M.out_fp32;
      float* dst32 = p.slices > 1 ? p.part_o + (orow * p.slices + slice) * D : reinterpret_cast<float*>(p.out) + orow * D;
#pragma unroll 1
      for (int c4 = 0; c4 < D / 32; ++c4) {
        uint32_t w[32];
        tmem_ld32(tO + c4 * 32, w);
        tc_wait_ld();
#pragma unroll
        for (int k = 0; k < 32; ++k) w[k] = __float_as_uint(__uint_as_float(w[k]) * inv);
        if (!ok || !row_here) {
        } else if (to_fp32) {
          uint4* dst = reinterpret_cast<uint4*>(dst32 + c4 * 32);
#pragma unroll
          for (int k = 0; k < 8; ++k) dst[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        } else {
          uint4* dst = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D + c4 * 32);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(__uint_as_float(w[8 * k + 2 * e]), __uint_as_float(w[8 * k + 2 * e + 1]));
            dst[k] = make_uint4(o[0], o[1], o[2], o[3]);
          }
        }
      }
      if (ok && row_here) {
        if (p.slices > 1) p.part_ml[orow * p.slices + slice] = make_float2(m_st, l_run);
        else if (p.lse) p.lse[orow] = some ? (m_st + log2f(l_run)) * 0.6931471805599453f : -INFINITY;
      }
    }
  }

  // ---- teardown: everyone is done with TMEM before it is released ----
  tc_fence_before();
  __syncthreads();
  if (warp == W_MMA) {
    if (issuer_stop[0] || issuer_stop[1]) __nanosleep(100000);  // (MMAs in flight that nobody waited for)
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TM_COLS) : "memory");
  }
}

template <int D>
cudaError_t launch(const PackedAttnParams& p, cudaStream_t s) {
  auto kern = packed_tile_kernel<D>;
  const cudaError_t e = hswa_prepare_kernel<packed_tile_kernel<D>>(kSmem);
  if (e != cudaSuccess) return e;
  // the softmax warps' request for registers is granted only if the launch gives the block 512 x 128
  static const cudaError_t budget = [&] {
    cudaFuncAttributes attr;
    const cudaError_t q = cudaFuncGetAttributes(&attr, kern);
    return q != cudaSuccess ? q : attr.numRegs < 128 ? cudaErrorLaunchOutOfResources : cudaSuccess;
  }();
  if (budget != cudaSuccess) return budget;
  kern<<<(unsigned)((int64_t)p.slices * p.m.Hkv * p.b.B * p.row_tiles), kThreads, kSmem, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t hswa_launch_packed_tile(const PackedAttnParams& p, cudaStream_t s) { return p.m.D == 128 ? launch<128>(p, s) : launch<64>(p, s); }
