// Attention over a 4-bit cache for few rows per KV head (single tokens, drafts: up to 32 tokens x query heads) over contexts of up to
// some thousand keys: hswa_packed_attn.
//
// A block per (request, KV head).  One warp fetches the pages' slabs (a bulk copy each: rows and scales lie together) into a ring of
// slots; every other warp takes whole 64-key tiles, with a softmax state of its own, and the block merges them at the end.
// Bound by HBM (0.5625 bytes per element) and, close behind, by the instructions that turn codes into fp16; so both products
// read their operands straight from the packed rows, without a trip through shared memory:
//   S^T [keys x rows] = K Q^T: the element order along D is free as long as K and Q agree, so lane (g, t) of the fragment takes
//     the t-th quarter of row g, contiguous: one load per row.  Scales multiply the fp16 values, which stay exact.
//   O^T [D x rows] += V^T P^T: a lane needs neighbouring KEYS of one element side by side.  It reads 16 (D = 128) or 8
//     neighbouring elements of two keys and exchanges nibbles: 4 logic instructions make 8 bytes of (key, key') pairs out of
//     two words, and each converts at once.
// Measured, 64 / 8 heads of 128, one token: 32 requests of 1000 keys 19 us, of 2000 29; 2 requests of up to 512 keys, 4 heads of 64: 7.5,
// bound by the chain from the length to the merge.
#include "packed_stream.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int TK = kStreamTile;
constexpr int NW = 7;   // warps that compute: with the producer two per scheduler, so that a block's threads get 128 or 255 registers
// slots of the ring, each K or V of a tile (K is done with half a tile earlier); with the sums of three warps, 2 blocks of up to
// 16 rows or one of 32 fill an SM
constexpr int slots_of(int nt) { return nt == 1 ? 21 : nt == 2 ? 18 : 36; }
constexpr int kThreads = (NW + 1) * 32;

template <int D>
constexpr int kSlotBytes = TK * (D / 2 + D / 16);

template <int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 4 ? 1 : 2) packed_decode_kernel(const PackedAttnParams p) {
  constexpr int NS = slots_of(NT);
  constexpr int ROW = D / 2, SC = D / 16, KS = D / 16, SLOT = kSlotBytes<D>;
  constexpr int COLS = 8 * NT;
  constexpr int MT = D / 16;                // 16-row tiles of O^T
  constexpr int STEP = D == 64 && NT < 4 ? TK : TK / NT;  // keys per softmax step (registers)
  constexpr int GROUPS = STEP / 16;
  extern __shared__ __align__(128) uint8_t smem[];
  float4* box = reinterpret_cast<float4*>(smem + NS * SLOT);               // [3][MT][NT][32] sums on their way
  uint2* s_q = reinterpret_cast<uint2*>(box + 3 * MT * NT * 32);           // [NT][KS][32] fragments of Q
  float* s_down = reinterpret_cast<float*>(s_q + NT * KS * 32);            // [COLS]
  float2* s_ml = reinterpret_cast<float2*>(s_down + COLS);                 // [NW][COLS]
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_ml + NW * COLS);          // full [NS], empty [NS]
  int* s_stop = reinterpret_cast<int*>(bars + 2 * NS);                     // a wait ran out
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;

  const uint32_t full0 = smem_u32(bars), empty0 = smem_u32(bars + NS);
  if (threadIdx.x < 2 * NS) {  // (full and empty lie side by side)
    mbar_init(full0 + 8 * threadIdx.x, 1);
    mbar_fence_init();
  }
  if (threadIdx.x == 0) *s_stop = 0;
  const int r = blockIdx.x / M.Hkv, kh = blockIdx.x % M.Hkv;
  // the producer's first page ids do not wait for the length (an id behind it goes unused)
  const int32_t* tbl = p.b.block_table + (int64_t)r * p.b.max_blocks;
  int ids_next = warp == NW && lane < p.b.max_blocks ? tbl[lane] : 0;
  const Stream sm = stream_of(p, r);
  __syncthreads();
  if (blockIdx.x == 0 && warp < NW) record_batch(p, NW * 32);  // (while the first tiles are on their way)
  if (sm.tiles == 0) return;

  const int slab = M.P * (ROW + SC);
  if (warp == NW) {
    // ======================= producer =======================
    const int ppt = TK / M.P;  // pages per tile: 1, 2 or 4
    bool ok = true;
    // K and V of two tiles at a time, a lane per page: waiting for a slot costs a few hundred cycles, and these waits overlap
    const int i = lane % ppt, kv = lane / ppt & 1, ahead = lane / (2 * ppt);
    const int n_pages = (sm.end + M.P - 1) / M.P;  // (0: a request without keys)
    int ids = 0;
    for (int j = 0; j < sm.tiles; j += 2) {
      if ((j * ppt & 31) == 0) {
        ids = ids_next;
        ids_next = j * ppt + 32 + lane < n_pages ? tbl[j * ppt + 32 + lane] : 0;
      }
      const int first = (j + ahead) * ppt, here = min(ppt, n_pages - first);  // pages of the lane's tile
      int page = __shfl_sync(0xffffffffu, ids, (first + i) & 31);
      const bool mine = ahead < 2 && j + ahead < sm.tiles;
      const int order = 2 * (j + ahead) + kv, slot = order % NS, round = order / NS;
      if (mine && round > 0) ok = mbar_wait(empty0 + 8 * slot, (round - 1) & 1);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) {
        if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 50);
        break;
      }
      if (mine && i == 0) mbar_arrive_expect_tx(full0 + 8 * slot, max(here, 0) * slab);
      __syncwarp();
      if (mine && i < here) {
        if (page < 0 || page >= p.num_pages) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, first + i, page);
          page = 0;
        }
        bulk_load(smem_u32(smem + slot * SLOT + i * slab), p.pool + (((int64_t)page * 2 + kv) * M.Hkv + kh) * slab, slab, full0 + 8 * slot);
      }
    }
    if (!ok) __nanosleep(100000);  // copies that nobody will wait for land before the block's memory is handed on
    return;
  }

  // ======================= consumers =======================
  const int kg = key_of(g), ka = key_of(2 * t), kb = key_of(2 * t + 1);
  // where the rows and scales of a 16-key group of a slot lie (a group is inside one page)
  const int page_shift = 31 - __clz(M.P), scales_at = M.P * ROW;
  auto rows_of = [&](int key0) { return (key0 >> page_shift) * slab + (key0 & (M.P - 1)) * ROW; };
  auto scales_of = [&](int key0) { return (key0 >> page_shift) * slab + scales_at + (key0 & (M.P - 1)) * SC; };
  auto consumers_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(NW * 32) : "memory"); };
  bool ok = true;
  const int rows = sm.n * M.G, end = sm.end;
  const int first_end = p.causal ? min(end, sm.len + 1) : end;  // keys that the first row sees
  auto has_row = [&](int tok) { return (unsigned)sm.t0 + (unsigned)tok < (unsigned)p.total_q; };

  // Q in fragment order, each row times its power of two: by every warp for itself, or by NT warps for all
  uint2 qf[NT == 1 ? KS : 1];
  float down1 = 0.f;
  if (NT == 1 || warp < NT) {
    const int col = (NT == 1 ? 0 : warp * 8) + g, tok = col / M.G;
    const bool there = col < rows && has_row(tok);
    uint4 wq[D / 32];  // the t-th quarter of the row: D / 4 elements
    const uint4* src = reinterpret_cast<const uint4*>(p.q + ((int64_t)(sm.t0 + tok) * M.Hq + kh * M.G + col % M.G) * D + t * (D / 4));
    float amax = 0.f;
#pragma unroll
    for (int k = 0; k < D / 32; ++k) wq[k] = there ? src[k] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const uint32_t u[4] = {wq[k].x, wq[k].y, wq[k].z, wq[k].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = unpack_bf16x2(u[e]);
        amax = finite_max(amax, f);
      }
    }
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    float up, down;
    q_powers(amax, &up, &down);
    down = fmaxf(down * p.scale_log2, 0x1p-126f);  // (never 0: a masked score stays minus infinity)
#pragma unroll
    for (int k = 0; k < D / 32; ++k) {
      const uint32_t u[4] = {wq[k].x, wq[k].y, wq[k].z, wq[k].w};
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float2 lo = unpack_bf16x2(u[2 * e]), hi = unpack_bf16x2(u[2 * e + 1]);
        const uint2 v = make_uint2(pack_half2(lo.x * up, lo.y * up), pack_half2(hi.x * up, hi.y * up));
        if constexpr (NT == 1) qf[2 * k + e] = v;
        else s_q[(warp * KS + 2 * k + e) * 32 + lane] = v;
      }
    }
    if constexpr (NT == 1) down1 = down;
    else if (t == 0) s_down[col] = down;
  }
  if constexpr (NT > 1) consumers_sync();

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
      mul[c][e] = NT == 1 ? __shfl_sync(0xffffffffu, down1, (2 * t + e) * 4) : s_down[col];
      see[c][e] = p.causal ? min(end, sm.len + col / M.G + 1) : end;
    }
  // the warp's tiles: every NW-th
  for (int j = warp; j < sm.tiles; j += NW) {
    const int k_at = 2 * j, k_slot = k_at % NS, v_slot = (k_at + 1) % NS;
    ok = __all_sync(0xffffffffu, mbar_wait(full0 + 8 * k_slot, (k_at / NS) & 1) && mbar_wait(full0 + 8 * v_slot, ((k_at + 1) / NS) & 1));
    if (!ok) {
      if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, r, j, 51);
      *reinterpret_cast<volatile int*>(s_stop) = 1;
      __nanosleep(100000);  // (copies in flight, as above)
      break;
    }
    const uint8_t *k_st = smem + k_slot * SLOT, *v_st = smem + v_slot * SLOT;
    const int pos0 = j * TK;
    const bool masked = pos0 + TK > first_end;
#pragma unroll 1
    for (int step = 0; step < TK / STEP; ++step) {
      if (step > 0 && masked && pos0 + step * STEP >= end) break;  // no keys behind here
      float S[GROUPS][NT][4];
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const uint8_t* rows_at = k_st + rows_of(step * STEP + q * 16);
        const uint8_t* sc_at = k_st + scales_of(step * STEP + q * 16);
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
      if (step + 1 == TK / STEP || (masked && pos0 + (step + 1) * STEP >= end)) {  // K has been read
        __syncwarp();
        if (lane == 0) mbar_arrive(empty0 + 8 * k_slot);
      }
      // masks, the running base of each row (column of S^T) in log2 units
      if (masked) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
#pragma unroll
          for (int q = 0; q < GROUPS; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (pos0 + step * STEP + q * 16 + kg + (e >> 1) * 8 >= see[c][e & 1]) S[q][c][e] = -INFINITY;
      }
      uint32_t P[GROUPS][NT][2];
#pragma unroll
      for (int c = 0; c < NT; ++c) {
        float mx[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[e] = fmaxf(S[0][c][e], S[0][c][e + 2]);
#pragma unroll
          for (int q = 1; q < GROUPS; ++q) mx[e] = max3(mx[e], S[q][c][e], S[q][c][e + 2]);
        }
#pragma unroll
        for (int sh = 4; sh <= 16; sh <<= 1) {
          mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], sh));
          mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], sh));
        }
        mx[0] = base_of(mx[0], mul[c][0]);
        mx[1] = base_of(mx[1], mul[c][1]);
        const bool grow0 = base_moves(mx[0], m[c][0]), grow1 = base_moves(mx[1], m[c][1]);
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
          const float e0 = fast_exp2(fmaf(S[q][c][0], mul[c][0], -mu0)), e1 = fast_exp2(fmaf(S[q][c][1], mul[c][1], -mu1)),
                      e2 = fast_exp2(fmaf(S[q][c][2], mul[c][0], -mu0)), e3 = fast_exp2(fmaf(S[q][c][3], mul[c][1], -mu1));
          l[c][0] += e0 + e2;
          l[c][1] += e1 + e3;
          P[q][c][0] = movmatrix_trans(pack_half2(e0, e1));
          P[q][c][1] = movmatrix_trans(pack_half2(e2, e3));
        }
      }
#pragma unroll
      for (int q = 0; q < GROUPS; ++q) {
        const uint8_t* rows_at = v_st + rows_of(step * STEP + q * 16);
        const uint8_t* sc_at = v_st + scales_of(step * STEP + q * 16);
        const int blk = D == 128 ? g : g >> 1;
        uint32_t f0 = sc_at[ka * SC + blk] | (uint32_t)sc_at[kb * SC + blk] << 8;
        uint32_t f1 = sc_at[(ka + 8) * SC + blk] | (uint32_t)sc_at[(kb + 8) * SC + blk] << 8;
        if (masked) {  // rows behind the last visible key hold anything, scales of NaN included: zero times their codes
          const int at = pos0 + step * STEP + q * 16;
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
    if (lane == 0) mbar_arrive(empty0 + 8 * v_slot);
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
  consumers_sync();
  if (*reinterpret_cast<volatile int*>(s_stop) != 0) return;
  float L[NT][2], top[NT][2];
#pragma unroll
  for (int c = 0; c < NT; ++c)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int col = c * 8 + 2 * t + e;
      float mm = -INFINITY;
#pragma unroll
      for (int k = 0; k < NW; ++k) mm = fmaxf(mm, s_ml[k * COLS + col].x);
      const float base = mm == -INFINITY ? 0.f : mm;
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float2 v = s_ml[k * COLS + col];
        sum += v.y != 0.f ? v.y * fast_exp2(v.x == -INFINITY ? 0.f : v.x - base) : 0.f;  // (l of NaN scores: m says nothing)
      }
      const float f = m[c][e] == -INFINITY ? 1.f : fast_exp2(m[c][e] - base);
      top[c][e] = mm;
      L[c][e] = sum;
      const float out = f * (sum != 0.f ? p.v_scale / sum : 0.f);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        O[i][c][e] *= out;
        O[i][c][e + 2] *= out;
      }
    }
  // the upper half of the warps hands its sums to the lower half, three times (same lane, same registers)
  static_assert(NW == 7, "three warps hand over at most");
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
      const int col = c * 8 + 2 * t + e, tok = col / M.G;
      if (col >= rows || !has_row(tok)) continue;
      const int64_t orow = (int64_t)(sm.t0 + tok) * M.Hq + kh * M.G + col % M.G;
      if (M.out_fp32) {
        float* dst = reinterpret_cast<float*>(p.out) + orow * D + g * (D / 8);
#pragma unroll
        for (int i = 0; i < MT; i += 2)
          *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(O[i][c][e], O[i][c][e + 2], O[i + 1][c][e], O[i + 1][c][e + 2]);
      } else {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D + g * (D / 8);
#pragma unroll
        for (int i = 0; i < MT; i += 4)
          *reinterpret_cast<uint4*>(dst + 2 * i) =
              make_uint4(pack_bf16x2(O[i][c][e], O[i][c][e + 2]), pack_bf16x2(O[i + 1][c][e], O[i + 1][c][e + 2]),
                         pack_bf16x2(O[i + 2][c][e], O[i + 2][c][e + 2]), pack_bf16x2(O[i + 3][c][e], O[i + 3][c][e + 2]));
      }
      if (g == 0 && p.lse) p.lse[orow] = L[c][e] != 0.f ? (top[c][e] + log2f(L[c][e])) * 0.6931471805599453f : -INFINITY;
    }
}

template <int D, int NT>
cudaError_t launch(const PackedAttnParams& p, cudaStream_t s) {
  constexpr int NS = slots_of(NT);
  constexpr int SMEM = NS * kSlotBytes<D> + 3 * D * NT * 32 + NT * D * 16 + 32 * NT + NW * 64 * NT + 16 * NS + 16;
  const cudaError_t e = hswa_prepare_kernel<packed_decode_kernel<D, NT>>(SMEM);
  if (e != cudaSuccess) return e;
  packed_decode_kernel<D, NT><<<p.b.B * p.m.Hkv, kThreads, SMEM, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t hswa_launch_packed_decode(const PackedAttnParams& p, int rows, cudaStream_t s) {
  if (p.m.D == 128) return rows == 8 ? launch<128, 1>(p, s) : rows == 16 ? launch<128, 2>(p, s) : launch<128, 4>(p, s);
  return rows == 8 ? launch<64, 1>(p, s) : rows == 16 ? launch<64, 2>(p, s) : launch<64, 4>(p, s);
}
