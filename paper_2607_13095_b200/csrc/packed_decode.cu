// Attention over a 4-bit cache for few rows per KV head (single tokens, drafts): hswa_packed_attn.
//
// A block takes one slice of a request's keys for one KV head and 8 NT rows (tokens x query heads).  One warp fetches the
// pages' slabs (a bulk copy each: rows and scales lie together) into a ring of 64-key stages; every other warp takes whole
// stages, with a softmax state of its own, and the block merges them at the end.  Bound by HBM (0.5625 bytes per element) and,
// close behind, by the instructions that turn codes into fp16; so both products read their operands straight from the packed
// rows, without a trip through shared memory:
//   S^T [keys x rows] = K Q^T: the element order along D is free as long as K and Q agree, so lane (g, t) of the fragment takes
//     the t-th quarter of row g, contiguous: one load per row.  Scales multiply the fp16 values, which stay exact.
//   O^T [D x rows] += V^T P^T: a lane needs neighbouring KEYS of one element side by side.  It reads 16 (D = 128) or 8
//     neighbouring elements of two keys and exchanges nibbles: 4 logic instructions make 8 bytes of (key, key') pairs out of
//     two words, and each converts at once.
#include "packed.cuh"

namespace {
using namespace hswa_dev;

constexpr int TK = 64;  // keys per stage
constexpr int NW = 7;   // warps that compute: with the producer two per scheduler, so that a block's threads get 128 or 255 registers
constexpr int NS = 12;  // stages
constexpr int kThreads = (NW + 1) * 32;

template <int D>
constexpr int kStageBytes = 2 * TK * (D / 2 + D / 16);

// Keys of a 16-key group in the order of the fragments' rows: row i of the first half holds key kKey(i), row 8 + i key 8 +
// kKey(i).  (A lane's V rows are kKey(2t), kKey(2t + 1): this order has lanes t = 0 .. 3 on rows 0, 3, 4, 7 and 1, 2, 5, 6,
// two of each parity, which halves the bank conflicts of 64-byte rows; K rows come in pairs of unlike parity.)
__device__ __forceinline__ int key_of(int i) { return (i & 4) | ((i & 2) ? 3 - (i & 1) : (i & 1)); }

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 4 ? 1 : 2) packed_decode_kernel(const PackedAttnParams p) {
  constexpr int ROW = D / 2, SC = D / 16, KS = D / 16, STAGE = kStageBytes<D>, HALF = STAGE / 2;
  constexpr int COLS = 8 * NT;
  constexpr int MT = D / 16;                // 16-row tiles of O^T
  constexpr int STEP = D == 64 && NT < 4 ? TK : TK / NT;  // keys per softmax step (registers)
  constexpr int GROUPS = STEP / 16;
  extern __shared__ __align__(128) uint8_t smem[];
  uint2* s_q = reinterpret_cast<uint2*>(smem + NS * STAGE);                 // [NT][KS][32] fragments of Q
  float* s_down = reinterpret_cast<float*>(s_q + NT * KS * 32);            // [COLS]
  float2* s_ml = reinterpret_cast<float2*>(s_down + COLS);                 // [NW][COLS]
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_ml + NW * COLS);          // full [NS], empty [NS]
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;

  const int r = blockIdx.x % p.b.B, rest = blockIdx.x / p.b.B;
  const int rt = rest % p.row_tiles, slice = rest / p.row_tiles, kh = blockIdx.y;
  const int t0 = p.b.q_indptr ? p.b.q_indptr[r] : r;
  const int n = p.b.q_indptr ? p.b.q_indptr[r + 1] - t0 : 1;
  const int ctx = p.b.ctx_len[r];
  if (threadIdx.x == 0 && rt == 0 && slice == 0 && kh == 0) {  // the grid was sized from the host's bounds
    if (ctx < 0 || ctx > p.max_ctx_len) record_error(p.err, HSWA_ERR_BOUNDS, r, -1, ctx);
    if (n < 0 || n > p.max_q_len || t0 < 0 || (int64_t)t0 + n > p.total_q) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, n);
  }
  const int len = max(0, min(ctx, p.max_ctx_len));
  auto has_row = [&](int tok) { return (unsigned)t0 + (unsigned)tok < (unsigned)p.total_q; };
  const int n_here = min(n, p.max_q_len);  // tokens that the grid covers
  if (p.slices > 1 && rt == 0 && slice == 0) {
    // rows past the host's bound have no block: a mark tells the join to leave them alone
    for (int64_t tok = (int64_t)p.max_q_len + threadIdx.x; tok < n; tok += kThreads)
      if (has_row((int)tok))
        for (int h = 0; h < M.G; ++h) p.part_ml[(((int64_t)t0 + tok) * M.Hq + kh * M.G + h) * p.slices] = make_float2(-INFINITY, -1.f);
  }
  const int row0 = rt * COLS, rows = n_here * M.G - row0;  // rows left from this block's first on
  if (rows <= 0) return;
  const int last_tok = (row0 + min(rows, COLS) - 1) / M.G;
  const int64_t room = (int64_t)p.b.max_blocks * M.P;  // positions that the block table has places for
  int end = p.causal ? len + last_tok + 1 : len;       // keys that the block's last row sees
  if (end > room) {
    if (threadIdx.x == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, -3, end);
    end = (int)room;
  }
  const int k0 = slice * p.slice_len;
  const int k1 = min(end, k0 + p.slice_len);
  const int tiles = k1 > k0 ? (k1 - k0 + TK - 1) / TK : 0;
  const int first_end = p.causal ? min(end, len + row0 / M.G + 1) : end;  // keys that its first row sees

  auto store_row = [&](int col, int d, const float* v, int count) {  // count = 8 or 16 neighbouring elements of a row
    const int row = row0 + col, tok = row / M.G;
    if (col >= rows || !has_row(tok)) return;
    const int64_t orow = (int64_t)(t0 + tok) * M.Hq + kh * M.G + row % M.G;
    if (p.slices > 1 || M.out_fp32) {
      float* dst = p.slices > 1 ? p.part_o + (orow * p.slices + slice) * D + d : reinterpret_cast<float*>(p.out) + orow * D + d;
      for (int k = 0; k < count; k += 4) *reinterpret_cast<float4*>(dst + k) = make_float4(v[k], v[k + 1], v[k + 2], v[k + 3]);
    } else {
      __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D + d;
      for (int k = 0; k < count; k += 8)
        *reinterpret_cast<uint4*>(dst + k) = make_uint4(pack_bf16x2(v[k], v[k + 1]), pack_bf16x2(v[k + 2], v[k + 3]),
                                                        pack_bf16x2(v[k + 4], v[k + 5]), pack_bf16x2(v[k + 6], v[k + 7]));
    }
  };
  auto store_ml = [&](int col, float m, float l) {
    const int row = row0 + col, tok = row / M.G;
    if (col >= rows || !has_row(tok)) return;
    const int64_t orow = (int64_t)(t0 + tok) * M.Hq + kh * M.G + row % M.G;
    if (p.slices > 1)
      p.part_ml[orow * p.slices + slice] = make_float2(m, l);
    else if (p.lse)
      p.lse[orow] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
  };

  if (tiles == 0) {  // no key here: zeros, or a partial that the join passes over
    const float zero[8] = {};
    for (int i = threadIdx.x; i < COLS; i += kThreads) store_ml(i, -INFINITY, 0.f);
    if (p.slices == 1)
      for (int i = threadIdx.x; i < COLS * D / 8; i += kThreads) store_row(i / (D / 8), i % (D / 8) * 8, zero, 8);
    return;
  }

  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + NS);
  if (threadIdx.x == 0) {
    for (int s = 0; s < NS; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    mbar_fence_init();
  }
  // Q: warp w < NT brings its eight rows into fragment order
  if (warp < NT) {
    const int col = warp * 8 + g, row = row0 + col, tok = row / M.G;
    const bool there = col < rows && has_row(tok);
    uint4 w[D / 32];  // the t-th quarter of the row: D / 4 elements
    const uint4* src = reinterpret_cast<const uint4*>(p.q + ((int64_t)(t0 + tok) * M.Hq + kh * M.G + row % M.G) * D + t * (D / 4));
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      w[k] = there ? src[k] : make_uint4(0, 0, 0, 0);
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack_bf16x2(u[e]);
        amax = fmaxf(amax, fmaxf(fabsf(f.x), fabsf(f.y)));
      }
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    float up, down;
    q_powers(amax, &up, &down);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const uint32_t u[4] = {w[k].x, w[k].y, w[k].z, w[k].w};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 lo = unpack_bf16x2(u[2 * e]), hi = unpack_bf16x2(u[2 * e + 1]);
        s_q[(warp * KS + 2 * k + e) * 32 + lane] = make_uint2(pack_half2(lo.x * up, lo.y * up), pack_half2(hi.x * up, hi.y * up));
      }
    }
    if (t == 0) s_down[col] = down * p.scale_log2;
  }
  __syncthreads();

  const int slab = M.P * (ROW + SC);
  if (warp == NW) {
    // ======================= producer =======================
    const int ppt = TK / M.P;  // pages per stage: 1, 2 or 4
    const int32_t* tbl = p.b.block_table + (int64_t)r * p.b.max_blocks + k0 / M.P;
    const int n_pages = (k1 - k0 + M.P - 1) / M.P;
    int ids_next = lane < n_pages ? tbl[lane] : 0, ids = 0;
    bool ok = true;
    for (int j = 0; j < tiles && ok; ++j) {
      const int stage = j % NS, first = j * ppt;
      if ((first & 31) == 0) {
        ids = ids_next;
        ids_next = first + 32 + lane < n_pages ? tbl[first + 32 + lane] : 0;
      }
      const int here = min(ppt, n_pages - first);  // pages of this stage
      const int i = lane % ppt, kv = lane / ppt;
      int page = __shfl_sync(0xffffffffu, ids, (first + i) & 31);
      if (j >= NS) ok = __all_sync(0xffffffffu, mbar_wait(empty0 + 8 * stage, ((j / NS) - 1) & 1));
      if (!ok) {
        if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 50);
        break;
      }
      if (lane == 0) mbar_arrive_expect_tx(full0 + 8 * stage, 2 * here * slab);
      __syncwarp();
      if (kv < 2 && i < here) {
        if (page < 0 || page >= p.num_pages) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, k0 / M.P + first + i, page);
          page = 0;
        }
        bulk_load(smem_u32(smem + stage * STAGE + kv * HALF + i * slab), p.pool + (((int64_t)page * 2 + kv) * M.Hkv + kh) * slab, slab,
                  full0 + 8 * stage);
      }
    }
    if (!ok) __nanosleep(100000);  // copies that nobody will wait for land before the block's memory is handed on
    return;
  }

  // ======================= consumers =======================
  float O[MT][NT][4];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int c = 0; c < NT; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) O[i][c][e] = 0.f;
  float m[NT][2], l[NT][2], mul[NT][2];
  int see[NT][2];  // keys that the lane's rows see (as positions)
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[c][e] = -INFINITY;
      l[c][e] = 0.f;
      const int col = c * 8 + 2 * t + e;
      mul[c][e] = s_down[col];
      see[c][e] = p.causal ? min(end, len + (row0 + col) / M.G + 1) : end;
    }
  uint2 qf[NT == 1 ? KS : 1];
  if constexpr (NT == 1) {
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[s] = s_q[s * 32 + lane];
  }
  const int kg = key_of(g), ka = key_of(2 * t), kb = key_of(2 * t + 1);
  bool ok = true;
  for (int j = warp; j < tiles; j += NW) {
    const int stage = j % NS;
    ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * stage, (j / NS) & 1));
    if (!ok) {
      if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 51);
      __nanosleep(100000);  // (copies in flight, as above)
      break;
    }
    const uint8_t* st = smem + stage * STAGE;
    const int pos0 = k0 + j * TK;
    const bool masked = pos0 + TK > first_end;
#pragma unroll
    for (int step = 0; step < TK / STEP; ++step) {
      if (masked && pos0 + step * STEP >= k1) break;  // nothing of the slice behind here
      float S[GROUPS][NT][4];
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const int key0 = step * STEP + q * 16, pg = key0 / M.P;
        const uint8_t* rows_at = st + pg * slab + (key0 - pg * M.P) * ROW;
        const uint8_t* sc_at = st + pg * slab + M.P * ROW + (key0 - pg * M.P) * SC;
        uint32_t wa[D / 32], wb[D / 32];
        uint32_t fa, fb;
        if constexpr (D == 128) {
          *reinterpret_cast<uint4*>(wa) = *reinterpret_cast<const uint4*>(rows_at + kg * ROW + t * 16);
          *reinterpret_cast<uint4*>(wb) = *reinterpret_cast<const uint4*>(rows_at + (kg + 8) * ROW + t * 16);
          fa = e4m3_to_half2(*reinterpret_cast<const uint16_t*>(sc_at + kg * SC + 2 * t));
          fb = e4m3_to_half2(*reinterpret_cast<const uint16_t*>(sc_at + (kg + 8) * SC + 2 * t));
        } else {
          *reinterpret_cast<uint2*>(wa) = *reinterpret_cast<const uint2*>(rows_at + kg * ROW + t * 8);
          *reinterpret_cast<uint2*>(wb) = *reinterpret_cast<const uint2*>(rows_at + (kg + 8) * ROW + t * 8);
          fa = e4m3_to_half2(sc_at[kg * SC + t]);
          fb = e4m3_to_half2(sc_at[(kg + 8) * SC + t]);
        }
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) S[q][c][e] = 0.f;
#pragma unroll
        for (int hf = 0; hf < D / 64; ++hf) {  // 16 elements of the lane's rows: one scale
          const uint32_t sa = hf ? high_twice(fa) : low_twice(fa), sb = hf ? high_twice(fb) : low_twice(fb);
#pragma unroll
          for (int s4 = 0; s4 < 4; ++s4) {
            const int s = hf * 4 + s4;
            const uint32_t ua = wa[s / 2], ub = wb[s / 2];
            const uint32_t a0 = hmul2((s & 1) ? e2m1_to_half2<2>(ua) : e2m1_to_half2<0>(ua), sa);
            const uint32_t a1 = hmul2((s & 1) ? e2m1_to_half2<2>(ub) : e2m1_to_half2<0>(ub), sb);
            const uint32_t a2 = hmul2((s & 1) ? e2m1_to_half2<3>(ua) : e2m1_to_half2<1>(ua), sa);
            const uint32_t a3 = hmul2((s & 1) ? e2m1_to_half2<3>(ub) : e2m1_to_half2<1>(ub), sb);
#pragma unroll
            for (int c = 0; c < NT; ++c) {
              const uint2 b = NT == 1 ? qf[NT == 1 ? s : 0] : s_q[(c * KS + s) * 32 + lane];
              mma_f16_16816(S[q][c], a0, a1, a2, a3, b.x, b.y);
            }
          }
        }
      }
      // scores in log2 units, masks, the running maximum of each row (column of S^T)
      uint32_t P[GROUPS][NT][2];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int q = 0; q < GROUPS; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = S[q][c][e] * mul[c][e & 1];
            if (masked && pos0 + step * STEP + q * 16 + kg + (e >> 1) * 8 >= see[c][e & 1]) x = -INFINITY;
            S[q][c][e] = x;
            mx[e & 1] = fmaxf(mx[e & 1], x);
          }
#pragma unroll
        for (int sh = 4; sh <= 16; sh <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], sh));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], sh));
        }
        // O moves to a new maximum only when that grew by more than 2^8 (P stays within fp16)
        const bool grow0 = mx[0] > m[c][0] + 8.f, grow1 = mx[1] > m[c][1] + 8.f;
        if (__any_sync(0xffffffffu, grow0 || grow1)) {
          const float al0 = grow0 ? fast_exp2(m[c][0] - mx[0]) : 1.f, al1 = grow1 ? fast_exp2(m[c][1] - mx[1]) : 1.f;
          if (grow0) m[c][0] = mx[0];
          if (grow1) m[c][1] = mx[1];
          l[c][0] *= al0;
          l[c][1] *= al1;
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            O[i][c][0] *= al0;
            O[i][c][1] *= al1;
            O[i][c][2] *= al0;
            O[i][c][3] *= al1;
          }
        }
        const float mu0 = m[c][0] == -INFINITY ? 0.f : m[c][0], mu1 = m[c][1] == -INFINITY ? 0.f : m[c][1];
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
          const float e0 = fast_exp2(S[q][c][0] - mu0), e1 = fast_exp2(S[q][c][1] - mu1), e2 = fast_exp2(S[q][c][2] - mu0),
                      e3 = fast_exp2(S[q][c][3] - mu1);
          l[c][0] += e0 + e2;
          l[c][1] += e1 + e3;
          P[q][c][0] = movmatrix_trans(pack_half2(e0, e1));
          P[q][c][1] = movmatrix_trans(pack_half2(e2, e3));
        }
      }
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const int key0 = step * STEP + q * 16, pg = key0 / M.P;
        const uint8_t* rows_at = st + HALF + pg * slab + (key0 - pg * M.P) * ROW;
        const uint8_t* sc_at = st + HALF + pg * slab + M.P * ROW + (key0 - pg * M.P) * SC;
        const int blk = D == 128 ? g : g >> 1;
        uint32_t f0 = sc_at[ka * SC + blk] | (uint32_t)sc_at[kb * SC + blk] << 8;
        uint32_t f1 = sc_at[(ka + 8) * SC + blk] | (uint32_t)sc_at[(kb + 8) * SC + blk] << 8;
        if (masked) {  // rows behind the last visible key hold anything, scales of NaN included: zero times their codes
          const int at = pos0 + key0;
          f0 &= (at + ka < end ? 0xffu : 0u) | (at + kb < end ? 0xff00u : 0u);
          f1 &= (at + ka + 8 < end ? 0xffu : 0u) | (at + kb + 8 < end ? 0xff00u : 0u);
        }
        const uint32_t s0 = e4m3_to_half2(f0), s1 = e4m3_to_half2(f1);
        uint32_t w[4][D / 64];
        const int keys[4] = {ka, kb, ka + 8, kb + 8};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (D == 128)
            *reinterpret_cast<uint2*>(w[k]) = *reinterpret_cast<const uint2*>(rows_at + keys[k] * ROW + g * 8);
          else
            w[k][0] = *reinterpret_cast<const uint32_t*>(rows_at + keys[k] * ROW + g * 4);
        }
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          constexpr uint32_t LOW = 0x0f0f0f0fu;
          const uint32_t ev0 = (w[0][x] & LOW) | ((w[1][x] << 4) & ~LOW), od0 = ((w[0][x] >> 4) & LOW) | (w[1][x] & ~LOW);
          const uint32_t ev1 = (w[2][x] & LOW) | ((w[3][x] << 4) & ~LOW), od1 = ((w[2][x] >> 4) & LOW) | (w[3][x] & ~LOW);
#define HSWA_PV(B)                                                                                                       \
  {                                                                                                                      \
    const uint32_t a0 = hmul2(e2m1_to_half2<B>(ev0), s0), a1 = hmul2(e2m1_to_half2<B>(od0), s0);                          \
    const uint32_t a2 = hmul2(e2m1_to_half2<B>(ev1), s1), a3 = hmul2(e2m1_to_half2<B>(od1), s1);                          \
    _Pragma("unroll") for (int c = 0; c < NT; ++c) mma_f16_16816(O[4 * x + B][c], a0, a1, a2, a3, P[q][c][0], P[q][c][1]); \
  }
          HSWA_PV(0) HSWA_PV(1) HSWA_PV(2) HSWA_PV(3)
#undef HSWA_PV
        }
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(empty0 + 8 * stage);
  }

  // ---- merge of the warps' states ----
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int sh = 4; sh <= 16; sh <<= 1) l[c][e] += __shfl_xor_sync(0xffffffffu, l[c][e], sh);
      if (g == 0) s_ml[warp * COLS + c * 8 + 2 * t + e] = make_float2(m[c][e], l[c][e]);
    }
  auto consumers_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(NW * 32) : "memory"); };
  consumers_sync();
  float L[NT][2], top[NT][2];
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int col = c * 8 + 2 * t + e;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < NW; ++w) mm = fmaxf(mm, s_ml[w * COLS + col].x);
      const float base = mm == -INFINITY ? 0.f : mm;
      float sum = 0.f;
#pragma unroll
      for (int w = 0; w < NW; ++w) {
        const float2 v = s_ml[w * COLS + col];
        sum += v.y != 0.f ? v.y * fast_exp2(v.x == -INFINITY ? 0.f : v.x - base) : 0.f;  // (l of NaN scores: m says nothing)
      }
      const float f = m[c][e] == -INFINITY ? 1.f : fast_exp2(m[c][e] - base);
      top[c][e] = mm;
      L[c][e] = sum;
      // the layer's V scale, and the division where the block has all of the row's keys
      const float out = f * (p.slices > 1 ? p.v_scale : (sum != 0.f ? p.v_scale / sum : 0.f));
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        O[i][c][e] *= out;
        O[i][c][e + 2] *= out;
      }
    }
  // the upper half of the warps hands its sums to the lower half, three times (same lane, same registers)
  float4* box = reinterpret_cast<float4*>(smem);
  static_assert(NW <= 8 && 4 * MT * NT * 32 * 16 <= NS * kStageBytes<D>, "sums fit the stages");
#pragma unroll
  for (int half = 4; half >= 1; half >>= 1) {
    if (warp >= half && warp < 2 * half) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < NT; ++c) box[(((warp - half) * MT + i) * NT + c) * 32 + lane] = make_float4(O[i][c][0], O[i][c][1], O[i][c][2], O[i][c][3]);
    }
    consumers_sync();
    if (warp < half && warp + half < NW) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int c = 0; c < NT; ++c) {
          const float4 v = box[((warp * MT + i) * NT + c) * 32 + lane];
          O[i][c][0] += v.x;
          O[i][c][1] += v.y;
          O[i][c][2] += v.z;
          O[i][c][3] += v.w;
        }
    }
    if (half > 1) consumers_sync();
  }
  if (warp != 0) return;
  // a lane holds D / 8 neighbouring elements of two rows per eight
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float v[2 * MT];
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        v[2 * i] = O[i][c][e];
        v[2 * i + 1] = O[i][c][e + 2];
      }
      const int col = c * 8 + 2 * t + e;
      store_row(col, g * (D / 8), v, D / 8);
      if (g == 0) store_ml(col, top[c][e], L[c][e]);
    }
}

template <int D, int NT>
cudaError_t launch(const PackedAttnParams& p, cudaStream_t s) {
  constexpr int SMEM = NS * kStageBytes<D> + NT * (D / 16) * 32 * 8 + 8 * NT * 4 + NW * 8 * NT * 8 + 2 * NS * 8;
  auto kern = packed_decode_kernel<D, NT>;
  const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
  if (e != cudaSuccess) return e;
  kern<<<dim3((unsigned)((int64_t)p.b.B * p.row_tiles * p.slices), p.m.Hkv, 1), kThreads, SMEM, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t hswa_launch_packed_decode(const PackedAttnParams& p, int rows, cudaStream_t s) {
  if (p.m.D == 128) return rows == 8 ? launch<128, 1>(p, s) : rows == 16 ? launch<128, 2>(p, s) : launch<128, 4>(p, s);
  return rows == 8 ? launch<64, 1>(p, s) : rows == 16 ? launch<64, 2>(p, s) : launch<64, 4>(p, s);
}
