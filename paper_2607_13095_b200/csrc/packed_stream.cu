// Attention over a 4-bit cache for up to eight rows per KV head (the single-token decode step): every warp on its own.
//
// The 64-key tiles of all (request, KV head) streams form one sequence, cut into equal runs, one per warp: no warp ends early,
// whatever the lengths, none waits for another, and loads run on from stream to stream.  A warp fetches its own tiles (a bulk copy
// per page and K or V) into a ring of its own, three half-tiles deep: V of the next tile is asked for when K of this one has been
// read, K of the one after when V has.  A stream that a warp has as a whole is written out there, pieces of the others are joined by
// a second launch.
// Both products read their operands straight from the packed rows, as in packed_decode.cu, which has the fragments' layout.
// Bound by HBM, and close behind by issue: of a 16-key group with 128 elements, the 64 conversions and 64 products that make fp16 of
// codes and the 16 MMAs take 240 of the 390 clocks that HBM leaves a scheduler, before loads, masks and the softmax.  Measured, 64 requests of one token over 4096 to
// 32768 keys, 64 / 8 heads of 128 (1.48 GB): 279 us, 5.3 TB/s (HBM floor 226); one warp that fetched for seven others 311, with
// divisions by the page size 365.
#include "packed_stream.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int TK = kStreamTile;
constexpr int NW = 8;  // warps of a block
constexpr int kThreads = NW * 32;

template <int D>
struct Cfg {
  static constexpr int ROW = D / 2, SC = D / 16, KS = D / 16, MT = D / 16;
  static constexpr int SLOT = TK * (ROW + SC);          // K or V of a tile
  static constexpr int SLOTS = D == 128 ? 3 : 6;        // of a warp; two blocks fill an SM
  static constexpr int SMEM = NW * SLOTS * (SLOT + 8) + 8 * (NW + 2 * NW);
};

// Where a warp is in its run.
struct Cursor {
  int r, kh, tile, left;  // request, KV head, tile of the stream, tiles left of the run
  Stream s;
};

template <int D, int PAGE>
__global__ void __launch_bounds__(kThreads, 2) packed_stream_kernel(const PackedAttnParams p) {
  using C = Cfg<D>;
  constexpr int ROW = C::ROW, SC = C::SC, KS = C::KS, MT = C::MT, SLOT = C::SLOT, SLOTS = C::SLOTS;
  constexpr int PPT = TK / PAGE, SLAB = PAGE * (ROW + SC);
  extern __shared__ __align__(128) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + NW * SLOTS * SLOT);  // [NW][SLOTS]
  int64_t* s_sums = reinterpret_cast<int64_t*>(bars + NW * SLOTS);         // [NW]
  int64_t* s_start = s_sums + NW;                                          // [NW][2] first request of a warp's run, tiles before it
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t = lane & 3;
  const int B = p.b.B;
  if (blockIdx.x == 0) record_batch(p, kThreads);
  const uint32_t bar0 = smem_u32(bars + warp * SLOTS), ring = smem_u32(smem) + warp * SLOTS * SLOT;
  const uint8_t* ring_ptr = smem + warp * SLOTS * SLOT;
  if (lane < SLOTS) mbar_init(bar0 + 8 * lane, 1);
  mbar_fence_init();

  // the warp's run of tiles [w0, w1) and where it starts
  int i0, i1;
  int64_t before;
  const int64_t heads = M.Hkv, total = sum_tiles<kThreads>(p, s_sums, &i0, &i1, &before) * heads;
  const int run = blockIdx.x * NW + warp;
  for (int i = i0; i < i1; ++i) {
    const int tiles = stream_of(p, i).tiles;
    if (blockIdx.x == 0) p.before[i] = before;  // for the join
    for (int k = 0; k < NW; ++k) {
      const int64_t x = blockIdx.x * NW + k < p.runs ? run_start(total, blockIdx.x * NW + k, p.runs) : -1;
      if (x >= before * heads && x < (before + tiles) * heads) {
        s_start[2 * k] = i;
        s_start[2 * k + 1] = before;
      }
    }
    before += tiles;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.before[B] = total / heads;
  __syncthreads();
  if (run >= p.runs) return;
  const int64_t w0 = run_start(total, run, p.runs), w1 = run_start(total, run + 1, p.runs);
  if (w0 >= w1) return;
  const int n_tiles = (int)(w1 - w0);
  Cursor at;
  at.r = (int)s_start[2 * warp];
  at.s = stream_of(p, at.r);
  at.kh = (int)((w0 - s_start[2 * warp + 1] * heads) / at.s.tiles);
  at.tile = (int)((w0 - s_start[2 * warp + 1] * heads) % at.s.tiles);
  at.left = n_tiles;
  // (requests with rows are left while tiles are)
  auto next_stream = [&](Cursor& c) {
    c.tile = 0;
    if (++c.kh == M.Hkv) {
      c.kh = 0;
      do {
        c.s = stream_of(p, ++c.r);
      } while (c.s.tiles == 0);
    }
  };

  // ---- fetching: K of the cursor's tile, then V of it, each into a slot that has just been read ----
  Cursor fc = at;
  const uint8_t* src = nullptr;  // K of the lane's page of the tile
  int here = 0;                  // pages of the tile
  const int64_t to_v = (int64_t)M.Hkv * SLAB;
  const int32_t* places = p.b.block_table + (int64_t)fc.r * p.b.max_blocks;
  auto load_page = [&](int tile) {
    const int place = tile * PPT + (PPT == 1 ? 0 : lane);
    return (PPT == 1 || lane < PPT) && place * PAGE < fc.s.end ? places[place] : 0;
  };
  int page = load_page(fc.tile);  // of the tile whose K comes next
  auto copy = [&](const uint8_t* from, uint32_t slot, uint32_t bar) {
    if (lane == 0) mbar_arrive_expect_tx(bar, max(here, 0) * SLAB);
    if constexpr (PPT == 1) {
      if (lane == 0 && here > 0) bulk_load(slot, from, SLAB, bar);
    } else {
      __syncwarp();
      if (lane < here) bulk_load(slot + lane * SLAB, from, SLAB, bar);
    }
  };
  auto fetch_k = [&](uint32_t slot, uint32_t bar) {
    if (fc.left == 0) return;
    here = min(PPT, (fc.s.end + PAGE - 1) / PAGE - fc.tile * PPT);
    if (page < 0 || page >= p.num_pages) {
      record_error(p.err, HSWA_ERR_BOUNDS, fc.r, fc.tile * PPT + (PPT == 1 ? 0 : lane), page);
      page = 0;
    }
    src = p.pool + ((int64_t)page * 2 * M.Hkv + fc.kh) * SLAB;
    page = load_page(fc.tile + 1);
    copy(src, slot, bar);
  };
  auto fetch_v = [&](uint32_t slot, uint32_t bar) {
    if (fc.left == 0) return;
    copy(src + to_v, slot, bar);
    --fc.left;
    if (++fc.tile == fc.s.tiles && fc.left > 0) {
      next_stream(fc);
      places = p.b.block_table + (int64_t)fc.r * p.b.max_blocks;
      page = load_page(0);
    }
  };
#pragma unroll 1
  for (int i = 0; i < SLOTS; i += 2) {
    fetch_k(ring + i * SLOT, bar0 + 8 * i);
    if (i + 1 < SLOTS) fetch_v(ring + (i + 1) * SLOT, bar0 + 8 * (i + 1));
  }

  const int kg = key_of(g), ka = key_of(2 * t), kb = key_of(2 * t + 1);
  int slot = 0;          // the next half-tile's slot and its barrier's phase
  uint32_t phase = 0;
  auto step = [&]() {
    if (++slot == SLOTS) {
      slot = 0;
      phase ^= 1;
    }
  };
  auto arrived = [&]() {  // (one poll where the copy has landed; the lanes may see it land at different polls, so each is voted on)
    const uint32_t bar = bar0 + 8 * slot;
    if (__all_sync(0xffffffffu, mbar_try_wait(bar, phase))) return true;
    return __all_sync(0xffffffffu, mbar_wait(bar, phase)) != 0;
  };
  auto give_up = [&]() {
    if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, at.r, at.tile, 52);
    __nanosleep(100000);  // copies that nobody will wait for land before the block's memory is handed on
  };
  while (at.left > 0) {
    // ---- a piece: the stream's tiles [at.tile, at.tile + count) ----
    const int count = min(at.s.tiles - at.tile, at.left), rows = at.s.n * M.G, end = at.s.end;
    const bool whole = count == at.s.tiles;
    const int first_end = p.causal ? min(end, at.s.len + 1) : end;  // keys that the first row sees
    auto has_row = [&](int tok) { return (unsigned)at.s.t0 + (unsigned)tok < (unsigned)p.total_q; };
    // Q in fragment order, each row times its power of two
    uint2 qf[KS];
    float down;
    {
      const int tok = g / M.G;
      const bool there = g < rows && has_row(tok);
      uint4 wq[D / 32];  // the t-th quarter of the row: D / 4 elements
      const uint4* src = reinterpret_cast<const uint4*>(p.q + ((int64_t)(at.s.t0 + tok) * M.Hq + at.kh * M.G + g % M.G) * D + t * (D / 4));
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
      float up;
      q_powers(amax, &up, &down);
      down = fmaxf(down * p.scale_log2, 0x1p-126f);  // (never 0: a masked score stays minus infinity)
#pragma unroll
      for (int k = 0; k < D / 32; ++k) {
        const uint32_t u[4] = {wq[k].x, wq[k].y, wq[k].z, wq[k].w};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float2 lo = unpack_bf16x2(u[2 * e]), hi = unpack_bf16x2(u[2 * e + 1]);
          qf[2 * k + e] = make_uint2(pack_half2(lo.x * up, lo.y * up), pack_half2(hi.x * up, hi.y * up));
        }
      }
    }
    float O[MT][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) O[i][e] = 0.f;
    float m[2], l[2], mul[2];
    int see[2];  // keys that the lane's rows see
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      m[e] = -INFINITY;
      l[e] = 0.f;
      mul[e] = __shfl_sync(0xffffffffu, down, (2 * t + e) * 4);
      see[e] = p.causal ? min(end, at.s.len + (2 * t + e) / M.G + 1) : end;
    }
#pragma unroll 1
    for (int j = 0; j < count; ++j) {
      const int pos0 = (at.tile + j) * TK;
      const bool masked = pos0 + TK > first_end;
      if (!arrived()) return give_up();
      const uint8_t* k_st = ring_ptr + slot * SLOT;
      float S[TK / 16][4];
#pragma unroll
      for (int q = 0; q < TK / 16; ++q) {
        const uint8_t* rows_at = k_st + q * 16 / PAGE * SLAB + q * 16 % PAGE * ROW;
        const uint8_t* sc_at = k_st + q * 16 / PAGE * SLAB + PAGE * ROW + q * 16 % PAGE * SC;
        uint32_t wa[D / 32], wb[D / 32], fa, fb;
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
            if (s == 0) mma_f16_16816_zero(S[q], a0, a1, a2, a3, qf[s].x, qf[s].y);
            else mma_f16_16816(S[q], a0, a1, a2, a3, qf[s].x, qf[s].y);
          }
        }
      }
      __syncwarp();
      if constexpr (SLOTS & 1) fetch_v(ring + slot * SLOT, bar0 + 8 * slot);
      else fetch_k(ring + slot * SLOT, bar0 + 8 * slot);
      step();
      // masks, the running base of each row (column of S^T) in log2 units
      if (masked) {
#pragma unroll
        for (int q = 0; q < TK / 16; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (pos0 + q * 16 + kg + (e >> 1) * 8 >= see[e & 1]) S[q][e] = -INFINITY;
      }
      float mx[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = fmaxf(S[0][e], S[0][e + 2]);
#pragma unroll
        for (int q = 1; q < TK / 16; ++q) mx[e] = max3(mx[e], S[q][e], S[q][e + 2]);
      }
#pragma unroll
      for (int sh = 4; sh <= 16; sh <<= 1) {
        mx[0] = fmaxf(mx[0], __shfl_xor_sync(0xffffffffu, mx[0], sh));
        mx[1] = fmaxf(mx[1], __shfl_xor_sync(0xffffffffu, mx[1], sh));
      }
      mx[0] = base_of(mx[0], mul[0]);
      mx[1] = base_of(mx[1], mul[1]);
      const bool grow0 = base_moves(mx[0], m[0]), grow1 = base_moves(mx[1], m[1]);
      if (__any_sync(0xffffffffu, grow0 || grow1)) {
        const float al0 = grow0 ? fast_exp2(m[0] - mx[0]) : 1.f, al1 = grow1 ? fast_exp2(m[1] - mx[1]) : 1.f;
        if (grow0) m[0] = mx[0];
        if (grow1) m[1] = mx[1];
        l[0] *= al0;
        l[1] *= al1;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          O[i][0] *= al0;
          O[i][1] *= al1;
          O[i][2] *= al0;
          O[i][3] *= al1;
        }
      }
      const float mu0 = m[0] == -INFINITY ? 0.f : m[0], mu1 = m[1] == -INFINITY ? 0.f : m[1];
      uint32_t P[TK / 16][2];
#pragma unroll
      for (int q = 0; q < TK / 16; ++q) {
        const float e0 = fast_exp2(fmaf(S[q][0], mul[0], -mu0)), e1 = fast_exp2(fmaf(S[q][1], mul[1], -mu1)),
                    e2 = fast_exp2(fmaf(S[q][2], mul[0], -mu0)), e3 = fast_exp2(fmaf(S[q][3], mul[1], -mu1));
        l[0] += e0 + e2;
        l[1] += e1 + e3;
        P[q][0] = movmatrix_trans(pack_half2(e0, e1));
        P[q][1] = movmatrix_trans(pack_half2(e2, e3));
      }
      if (!arrived()) return give_up();
      const uint8_t* v_st = ring_ptr + slot * SLOT;
#pragma unroll
      for (int q = 0; q < TK / 16; ++q) {
        const uint8_t* rows_at = v_st + q * 16 / PAGE * SLAB + q * 16 % PAGE * ROW;
        const uint8_t* sc_at = v_st + q * 16 / PAGE * SLAB + PAGE * ROW + q * 16 % PAGE * SC;
        const int blk = D == 128 ? g : g >> 1;
        uint32_t f0 = sc_at[ka * SC + blk] | (uint32_t)sc_at[kb * SC + blk] << 8;
        uint32_t f1 = sc_at[(ka + 8) * SC + blk] | (uint32_t)sc_at[(kb + 8) * SC + blk] << 8;
        if (masked) {  // rows behind the last visible key hold anything, scales of NaN included: zero times their codes
          const int pos = pos0 + q * 16;
          f0 &= (pos + ka < end ? 0xffu : 0u) | (pos + kb < end ? 0xff00u : 0u);
          f1 &= (pos + ka + 8 < end ? 0xffu : 0u) | (pos + kb + 8 < end ? 0xff00u : 0u);
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
#define HSWA_PV(b)                                                                                                        \
  mma_f16_16816(O[4 * x + b], hmul2(e2m1_to_half2<b>(ev0), s0), hmul2(e2m1_to_half2<b>(od0), s0), hmul2(e2m1_to_half2<b>(ev1), s1), \
                hmul2(e2m1_to_half2<b>(od1), s1), P[q][0], P[q][1]);
          HSWA_PV(0) HSWA_PV(1) HSWA_PV(2) HSWA_PV(3)
#undef HSWA_PV
        }
      }
      __syncwarp();
      if constexpr (SLOTS & 1) fetch_k(ring + slot * SLOT, bar0 + 8 * slot);
      else fetch_v(ring + slot * SLOT, bar0 + 8 * slot);
      step();
    }

    // ---- the piece's end ----
    const int64_t piece = 2 * (int64_t)run + (at.tile == 0);  // a run has one piece at most that starts before it, and one that ends behind it
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
      for (int sh = 4; sh <= 16; sh <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], sh);
      const int col = 2 * t + e, tok = col / M.G;
      if (col >= rows || !has_row(tok)) continue;
      const float f = !whole ? p.v_scale : (l[e] != 0.f ? p.v_scale / l[e] : 0.f);  // (a NaN among the inputs shows in the output)
      const int64_t orow = (int64_t)(at.s.t0 + tok) * M.Hq + at.kh * M.G + col % M.G;
      // a lane holds D / 8 neighbouring elements of its rows
      if (!whole || M.out_fp32) {
        float* dst = (!whole ? p.part_o + (piece * 8 + col) * D : reinterpret_cast<float*>(p.out) + orow * D) + g * (D / 8);
#pragma unroll
        for (int i = 0; i < MT; i += 2)
          *reinterpret_cast<float4*>(dst + 2 * i) = make_float4(O[i][e] * f, O[i][e + 2] * f, O[i + 1][e] * f, O[i + 1][e + 2] * f);
      } else {
        __nv_bfloat16* dst = reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D + g * (D / 8);
#pragma unroll
        for (int i = 0; i < MT; i += 4)
          *reinterpret_cast<uint4*>(dst + 2 * i) =
              make_uint4(pack_bf16x2(O[i][e] * f, O[i][e + 2] * f), pack_bf16x2(O[i + 1][e] * f, O[i + 1][e + 2] * f),
                         pack_bf16x2(O[i + 2][e] * f, O[i + 2][e + 2] * f), pack_bf16x2(O[i + 3][e] * f, O[i + 3][e + 2] * f));
      }
      if (g == 0) {
        if (!whole) p.part_ml[piece * 8 + col] = make_float2(m[e], l[e]);
        else if (p.lse) p.lse[orow] = l[e] != 0.f ? (m[e] + log2f(l[e])) * 0.6931471805599453f : -INFINITY;
      }
    }
    at.left -= count;
    at.tile += count;
    if (at.left > 0) next_stream(at);
  }
}

// Joins the pieces of the streams that several warps or blocks had: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
// ROWS = 8: eight rows of a stream per block, a warp each, or all warps on one after the other where the stream is in many pieces;
// 1: all warps on one row, for calls whose streams are all in many.  (32 requests of 4 tokens and 600 to 1500 keys, 64 / 8 heads, two or
// three pieces a stream: 10 us; 30 us with a block per row, most of which found nothing to do but to read where the runs begin.)
template <int D, int TILE, int ROWS>
__global__ void __launch_bounds__(256) packed_join_kernel(const PackedAttnParams p, const int cols) {
  const ModelParams& M = p.m;
  const int r = blockIdx.x / M.Hkv, kh = blockIdx.x % M.Hkv;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const Stream s = stream_of<TILE>(p, r);
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched early behind the kernel that writes the pieces
  const int64_t total = p.before[p.b.B] * M.Hkv, start = p.before[r] * M.Hkv + (int64_t)kh * s.tiles;
  const int rows = s.n * M.G;
  if (s.tiles == 0 || (int)blockIdx.y * ROWS >= rows) return;
  // run c holds tile x: c = ceil((x + 1) runs / total) - 1
  const int c0 = (int)(((start + 1) * p.runs - 1) / total), c1 = (int)(((start + s.tiles) * p.runs - 1) / total);
  if (c0 == c1) return;
  constexpr int PER = D / 32;
  __shared__ float sums[8][32][PER + 1];
  // the row's pieces first, first + step, ...: their sums under the row's maximum
  auto add_up = [&](int col, int first, int step, float (&acc)[PER], float& L) {
    auto piece_of = [&](int c) { return (2 * (int64_t)c + (c == c0)) * cols + col; };
    // a run without tiles (there may be more runs than tiles) left no piece; nor has a piece without a key of the row anything (l = 0)
    auto ml_of = [&](int c) {
      return p.runs <= total || run_start(total, c, p.runs) < run_start(total, c + 1, p.runs) ? p.part_ml[piece_of(c)]
                                                                                               : make_float2(-INFINITY, 0.f);
    };
    float mm = -INFINITY;
    for (int c = c0 + lane; c <= c1; c += 32) {
      const float2 v = ml_of(c);
      if (v.y != 0.f) mm = fmaxf(mm, v.x);
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, sh));
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = 0.f;
    L = 0.f;
#pragma unroll 4
    for (int c = c0 + first; c <= c1; c += step) {
      const float2 v = ml_of(c);
      const float f = v.y != 0.f ? fast_exp2(v.x == -INFINITY ? 0.f : v.x - mm) : 0.f;  // (l of NaN scores: m says nothing)
      const float* o = p.part_o + piece_of(c) * D + lane * PER;
      L += v.y != 0.f ? f * v.y : 0.f;
#pragma unroll
      for (int i = 0; i < PER; i += 2) {
        const float2 x = *reinterpret_cast<const float2*>(o + i);
        acc[i] += v.y != 0.f ? f * x.x : 0.f;
        acc[i + 1] += v.y != 0.f ? f * x.y : 0.f;
      }
    }
    return mm;
  };
  auto store = [&](int col, float mm, const float (&acc)[PER], float L) {
    const int tok = col / M.G;
    if ((unsigned)s.t0 + (unsigned)tok >= (unsigned)p.total_q) return;
    const float inv = L != 0.f ? 1.f / L : 0.f;
    const int64_t orow = (int64_t)(s.t0 + tok) * M.Hq + kh * M.G + col % M.G;
#pragma unroll
    for (int i = 0; i < PER; i += 2) {
      const int64_t at = orow * D + lane * PER + i;
      if (M.out_fp32)
        *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + at) = make_float2(acc[i] * inv, acc[i + 1] * inv);
      else
        *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at) = __floats2bfloat162_rn(acc[i] * inv, acc[i + 1] * inv);
    }
    if (lane == 0 && p.lse) p.lse[orow] = L != 0.f ? (mm + log2f(L)) * 0.6931471805599453f : -INFINITY;
  };
  float acc[PER], L;
  if (ROWS == 8 && c1 - c0 < 24) {
    const int col = blockIdx.y * 8 + warp;
    if (col >= rows) return;
    const float mm = add_up(col, 0, 1, acc, L);
    store(col, mm, acc, L);
    return;
  }
  for (int k = 0; k < ROWS; ++k) {
    const int col = blockIdx.y * ROWS + k;
    if (col >= rows) break;  // (uniform)
    const float mm = add_up(col, warp, 8, acc, L);
#pragma unroll
    for (int i = 0; i < PER; ++i) sums[warp][lane][i] = acc[i];
    sums[warp][lane][PER] = L;
    __syncthreads();
    if (warp == 0) {
#pragma unroll
      for (int w = 1; w < 8; ++w) {
#pragma unroll
        for (int i = 0; i < PER; ++i) acc[i] += sums[w][lane][i];
        L += sums[w][lane][PER];
      }
      store(col, mm, acc, L);
    }
    __syncthreads();
  }
}

template <int D, int PAGE>
cudaError_t launch(const PackedAttnParams& p, cudaStream_t s) {
  const cudaError_t e = hswa_prepare_kernel<packed_stream_kernel<D, PAGE>>(Cfg<D>::SMEM);
  if (e != cudaSuccess) return e;
  packed_stream_kernel<D, PAGE><<<(p.runs + NW - 1) / NW, kThreads, Cfg<D>::SMEM, s>>>(p);
  return cudaGetLastError();
}
template <int D>
cudaError_t launch(const PackedAttnParams& p, cudaStream_t s) {
  return p.m.P == 64 ? launch<D, 64>(p, s) : p.m.P == 32 ? launch<D, 32>(p, s) : launch<D, 16>(p, s);
}

}  // namespace

int hswa_packed_stream_runs_per_sm() { return 2 * NW; }

cudaError_t hswa_launch_packed_stream(const PackedAttnParams& p, cudaStream_t s) {
  const cudaError_t e = p.m.D == 128 ? launch<128>(p, s) : launch<64>(p, s);
  return e != cudaSuccess ? e : hswa_launch_packed_join(p, 8, TK, s);
}

template <int D, int TILE>
static cudaError_t launch_join(const PackedAttnParams& p, int cols, cudaStream_t s) {
  const int streams = p.b.B * p.m.Hkv, rows = p.max_q_len * p.m.G;
  const bool few = p.runs <= 8LL * streams;  // pieces of a stream, on the average
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(streams, few ? (rows + 7) / 8 : rows, 1);
  cfg.blockDim = dim3(256, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return few ? cudaLaunchKernelEx(&cfg, packed_join_kernel<D, TILE, 8>, p, cols) : cudaLaunchKernelEx(&cfg, packed_join_kernel<D, TILE, 1>, p, cols);
}
cudaError_t hswa_launch_packed_join(const PackedAttnParams& p, int cols, int tile, cudaStream_t s) {
  if (tile == TK) return p.m.D == 128 ? launch_join<128, TK>(p, cols, s) : launch_join<64, TK>(p, cols, s);
  return p.m.D == 128 ? launch_join<128, 128>(p, cols, s) : launch_join<64, 128>(p, cols, s);
}
