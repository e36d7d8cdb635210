// Attention over a 4-bit cache for few rows per KV head (up to 32 tokens x query heads) over long contexts on the 5th-generation
// tensor cores: hswa_packed_attn.
//
// The 128-key tiles of all (request, KV head) streams form one sequence, cut into equal runs, one per SM: no block ends early,
// whatever the lengths.  The keys are the MMAs' 128 rows and the query rows their N columns, so no product is spent on rows that
// are not there:
//   S^T [128 keys x N] = K Q^T    A = K from TMEM, B = Q from shared memory
//   O^T [D x N] += V^T P^T        A = V from shared memory ([key][element], the MMA transposes), B = P from shared memory
// Warp roles:
//   0-3    unpack K: codes and scales to fp16 in TMEM, four lanes per key (the order of the elements along D is free as long as Q's is
//          the same)
//   4-7    unpack V into swizzled shared memory
//   8-15   softmax, two groups of four warps with every second tile, each with maxima, sums and an accumulator of O of its own: TMEM
//          lane = key; a lane has N scores of its key.  The rows' bases (packed.cuh) are kept from tile to tile and moved only when a score passes
//          one by more than 2^15, which a vote over the four warps finds out; row sums stay in the lanes to the end
//   16-19  issue the MMAs of S, issue those of O, bring Q of the next stream, and fetch the tiles to come into a ring (a TMA load for
//          both slabs of a page)
// HBM would allow 790 clocks a tile at a head dim of 128; a tile takes 1300 with 16 columns and 1600 with 32, bound by the chain of
// each role's steps rather than by a pipe: every scheduler has five warps, half of its issue slots go unused.  Measured, 64 / 8 heads of
// 128, 32 requests of 4096 to 32768 keys: 2 tokens each 185 us, 2 to 4 tokens 245 us (HBM floor 98), where warp-level MMAs took 267 and
// 450.  Also tried: one softmax group 325 us; codes read straight from global memory 370; a descriptor ring with a prefetch to L2 328.
#include "packed_stream.cuh"
#include "tc_primitives.cuh"

namespace {
using namespace hswa_dev;

constexpr int TN = 128;  // keys per tile
constexpr int kThreads = 640;
constexpr int W_V = 4, W_SOFTMAX = 8, W_OTHER = 16;
// Registers per thread once the roles have split: their sum is what the launch gave (640 x 96).  32 scores of a lane want more of
// them than 16 (drafts of 32 rows below: 259 us with the first split, 245 with the second; of 16 rows 185 and 190).
template <int N>
struct Regs {
  static constexpr int K = N == 16 ? 88 : 80, V = 72, SOFTMAX = N == 16 ? 136 : 144, OTHER = N == 16 ? 48 : 40;
  static_assert(K + V + 2 * SOFTMAX + OTHER == 5 * 96, "what the launch gave");
};
constexpr int K_STAGES = 3, V_STAGES = 2;
constexpr int RING = 5;  // tiles of packed rows

constexpr int HALF_BYTES = TN * 128;  // 64 elements of each of a tile's rows
constexpr int V_BYTES = 2 * HALF_BYTES, P_BYTES = HALF_BYTES;
constexpr int TM_S = 192, TM_O = 256, TM_COLS = 512;  // TMEM: K stages, S [group], O [piece][group]

enum { B_KFULL = 0, B_KEMPTY = 3, B_VFULL = 6, B_VEMPTY = 9, B_SFULL = 12, B_SFREE = 14, B_PFULL = 16, B_PEMPTY = 18, B_QFULL = 20, B_QFREE = 22,
       B_OFULL = 24 /* [piece][group] */, B_OFREE = 28, B_RFULL = 32, B_REMPTY = B_RFULL + RING, NBARS = B_REMPTY + RING };

template <int D, int N>
struct Smem {
  static constexpr int Q_BYTES = N * 256;
  static constexpr int PACKED = TN * (D / 2 + D / 16);  // K or V of a tile
  static constexpr int OFF_V = 0, OFF_P = V_STAGES * V_BYTES, OFF_Q = OFF_P + 2 * P_BYTES, OFF_RING = OFF_Q + 2 * Q_BYTES;
  static constexpr int OFF_STATE = OFF_RING + RING * 2 * PACKED;
  static_assert(OFF_RING % 128 == 0 && PACKED % 128 == 0, "TMA destinations");
  static constexpr int GROUP_STATE = 6 * N * 4;  // of a softmax group: bases by warp [4][N], of the rows [N], factors of O [N]
  static constexpr int OFF_BARS = OFF_STATE + 2 * GROUP_STATE;
  static constexpr int OFF_PLAN = OFF_BARS + NBARS * 8;  // sums [20], first request, tiles before it
  static constexpr int OFF_MISC = OFF_PLAN + 22 * 8;     // TMEM base, a spare word, multiplier [4], keys of the ring's tiles [RING]
  static constexpr int BYTES = OFF_MISC + 24 + 4 * RING;
};

__device__ __forceinline__ void tmem_st_16x256b_x8(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x8.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
      "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
      : "memory");
}
__device__ __forceinline__ void tmem_st_16x256b_x4(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.16x256b.x4.b32 [%16], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::"r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
      "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr)
      : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_ld_cols(uint32_t addr, uint32_t* r) {
  if constexpr (N == 32) tmem_ld32(addr, r);
  else tmem_ld16(addr, r);
}
template <int N>
__device__ __forceinline__ void tmem_st_cols(uint32_t addr, const uint32_t* r) {
  if constexpr (N == 32) tmem_st32(addr, r);
  else tmem_st16p(addr, r);
}
// A bounded wait in as few instructions as it can be polled with: twenty warps share the SM, and what the waiting ones issue the
// others cannot (reading the clock at each poll, and a hint to sleep, took near half of all issue slots).  It gives up after 2^19
// polls, each of which suspends the thread for some 8000 clocks (measured on a barrier that nothing completes): two seconds.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, 0;\n"
      "POLL:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t@p bra DONE;\n\t"
      "add.u32 n, n, 1;\n\tsetp.lt.u32 q, n, 524288;\n\t@q bra POLL;\n"
      "DONE:\n\tselp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// The largest over the warp (NaN are passed over).
__device__ __forceinline__ float warp_max(float x) {
  float r;
  asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// Does the predicate hold for a thread of the four warps of softmax group `group`?
__device__ __forceinline__ bool softmax_any(int group, bool pred) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, %2, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(any)
               : "r"((uint32_t)pred), "r"(1 + group)
               : "memory");
  return any != 0;
}
// The same over both groups.
__device__ __forceinline__ bool groups_any(bool pred) {
  uint32_t any;
  asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 3, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
               : "=r"(any)
               : "r"((uint32_t)pred)
               : "memory");
  return any != 0;
}
__device__ __forceinline__ void softmax_sync(int group) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(1 + group) : "memory"); }

// A role's place in the block's run of tiles.
struct Walk {
  int r, kh, tile, left;  // request, KV head, tile of the stream, tiles left of the run
  Stream s;
  __device__ __forceinline__ int count() const { return min(s.tiles - tile, left); }  // tiles of this piece left
  // on to the next piece (requests with rows are left while tiles are)
  __device__ __forceinline__ void next_stream(const PackedAttnParams& p) {
    tile = 0;
    if (++kh == p.m.Hkv) {
      kh = 0;
      do s = stream_of<TN>(p, ++r); while (s.tiles == 0);
    }
  }
};

template <int D, int N>
__global__ void __launch_bounds__(kThreads, 1) packed_rows_kernel(const __grid_constant__ CUtensorMap tm_pool, const PackedAttnParams p) {
  using L = Smem<D, N>;
  constexpr int ROW = D / 2, SC = D / 16;
  constexpr int K_COLS = D / 2;  // TMEM columns of a K stage
  constexpr uint32_t IDESC_S = (1u << 4) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(TN >> 4) << 24);
  constexpr uint32_t IDESC_O = IDESC_S | (1u << 15) | (1u << 16);  // both operands [key][...]: transposed
  extern __shared__ __align__(1024) uint8_t smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BARS);
  int64_t* s_plan = reinterpret_cast<int64_t*>(smem + L::OFF_PLAN);
  uint32_t& s_tmem = *reinterpret_cast<uint32_t*>(smem + L::OFF_MISC);
  int* s_valid = reinterpret_cast<int*>(smem + L::OFF_MISC + 24);
  // from a raw score to log2 units, of a piece: Q may be brought up to three pieces before the softmax warps are there
  volatile float* s_mul = reinterpret_cast<volatile float*>(smem + L::OFF_MISC + 8);  // [4]
  const ModelParams& M = p.m;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t sbase = smem_u32(smem);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };

  if (blockIdx.x == 0) record_batch(p, kThreads);
  if (threadIdx.x == 0) {
    for (int i = 0; i < K_STAGES; ++i) {
      mbar_init(bar(B_KFULL + i), 4);
      mbar_init(bar(B_KEMPTY + i), 1);
    }
    for (int i = 0; i < V_STAGES; ++i) {
      mbar_init(bar(B_VFULL + i), 4);
      mbar_init(bar(B_VEMPTY + i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(B_SFULL + i), 1);
      mbar_init(bar(B_SFREE + i), 4);
      mbar_init(bar(B_PFULL + i), 4);
      mbar_init(bar(B_PEMPTY + i), 1);
      mbar_init(bar(B_QFULL + i), 1);
      mbar_init(bar(B_QFREE + i), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(B_OFULL + i), 1);
      mbar_init(bar(B_OFREE + i), 4);
    }
    for (int i = 0; i < RING; ++i) {
      mbar_init(bar(B_RFULL + i), 1);
      mbar_init(bar(B_REMPTY + i), 8);  // the unpacking warps
    }
    mbar_fence_init();
  }
  // the block's run of tiles [w0, w1), and where it starts
  int i0, i1;
  int64_t before;
  const int64_t heads = M.Hkv, total = sum_tiles<kThreads, TN>(p, s_plan, &i0, &i1, &before) * heads;
  const int64_t w0 = run_start(total, blockIdx.x, p.runs), w1 = run_start(total, blockIdx.x + 1, p.runs);
  for (int i = i0; i < i1; ++i) {
    const int tiles = stream_of<TN>(p, i).tiles;
    if (blockIdx.x == 0) p.before[i] = before;  // for the join
    if (w0 >= before * heads && w0 < (before + tiles) * heads) {
      s_plan[20] = i;
      s_plan[21] = before;
    }
    before += tiles;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) p.before[p.b.B] = total / heads;
  if constexpr (D == 64) {  // the MMA's rows behind the 64 elements are zeros
    for (int i = threadIdx.x; i < V_STAGES * HALF_BYTES / 16; i += kThreads)
      *reinterpret_cast<uint4*>(smem + L::OFF_V + i / (HALF_BYTES / 16) * V_BYTES + HALF_BYTES + i % (HALF_BYTES / 16) * 16) = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  if (warp == W_OTHER) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(TM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const int n_tiles = (int)(w1 - w0);
  Walk at = {};
  if (n_tiles > 0) {
    at.r = (int)s_plan[20];
    at.s = stream_of<TN>(p, at.r);
    at.kh = (int)((w0 - s_plan[21] * heads) / at.s.tiles);
    at.tile = (int)((w0 - s_plan[21] * heads) % at.s.tiles);
    at.left = n_tiles;
  }
  const int slab = M.P * (ROW + SC);
  auto timed_out = [&](int who, int i) {
    if (lane == 0) record_error(p.err, HSWA_ERR_TIMEOUT, blockIdx.x, i, who);
  };

  if (warp < W_V) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Regs<N>::K) : "memory");
    // ======================= unpack K =======================
    // Lane (g, t) takes the t-th quarter of rows 32 warp + 16 half + {g, g + 8}.
    const int g = lane >> 2, t = lane & 3;
    int at_rows[2], at_scales[2];  // where its rows and scales lie in the ring's tile
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const int key = warp * 32 + hf * 16 + g, slot = key & (M.P - 1), in_page = (key - slot) / M.P * 2 * slab;
      at_rows[hf] = in_page + slot * ROW + t * (D / 8);
      at_scales[hf] = in_page + M.P * ROW + slot * SC + t * (D / 64);
    }
    bool ok = true;
    for (int i = 0; i < n_tiles && ok; ++i) {
      const int stage = i % K_STAGES, rs = i % RING;
      ok = __all_sync(0xffffffffu, wait_for(bar(B_RFULL + rs), (i / RING) & 1));
      const uint8_t* tile = smem + L::OFF_RING + rs * 2 * L::PACKED;
      uint32_t data[2][2][D / 32], f[2][2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint8_t *rows = tile + at_rows[hf] + 8 * e * ROW, *scales = tile + at_scales[hf] + 8 * e * SC;
          if constexpr (D == 128) {
            const uint4 v = *reinterpret_cast<const uint4*>(rows);
            data[hf][e][0] = v.x, data[hf][e][1] = v.y, data[hf][e][2] = v.z, data[hf][e][3] = v.w;
            f[hf][e] = *reinterpret_cast<const uint16_t*>(scales);
          } else {
            const uint2 v = *reinterpret_cast<const uint2*>(rows);
            data[hf][e][0] = v.x, data[hf][e][1] = v.y;
            f[hf][e] = *scales;
          }
        }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_REMPTY + rs));
      if (i >= K_STAGES && !__all_sync(0xffffffffu, wait_for(bar(B_KEMPTY + stage), (i / K_STAGES - 1) & 1))) ok = false;
      if (!ok) break;
      tc_fence_after();
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        uint32_t o[D / 4];  // 256-bit blocks of 16 rows: (row g, columns 2t, 2t + 1), (row g + 8, the same)
        const uint32_t f0 = e4m3_to_half2(f[hf][0]), f1 = e4m3_to_half2(f[hf][1]);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          const uint32_t s0 = j < 4 ? low_twice(f0) : high_twice(f0), s1 = j < 4 ? low_twice(f1) : high_twice(f1);
          const uint32_t a = data[hf][0][j / 2], b = data[hf][1][j / 2];
          o[4 * j + 0] = hmul2((j & 1) ? e2m1_to_half2<2>(a) : e2m1_to_half2<0>(a), s0);
          o[4 * j + 1] = hmul2((j & 1) ? e2m1_to_half2<3>(a) : e2m1_to_half2<1>(a), s0);
          o[4 * j + 2] = hmul2((j & 1) ? e2m1_to_half2<2>(b) : e2m1_to_half2<0>(b), s1);
          o[4 * j + 3] = hmul2((j & 1) ? e2m1_to_half2<3>(b) : e2m1_to_half2<1>(b), s1);
        }
        const uint32_t to = tmem + ((uint32_t)(warp * 32 + hf * 16) << 16) + stage * K_COLS;
        if constexpr (D == 128) tmem_st_16x256b_x8(to, o);
        else tmem_st_16x256b_x4(to, o);
      }
      tc_wait_st();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_KFULL + stage));
    }
    if (!ok) timed_out(70, 0);
  } else if (warp < W_SOFTMAX) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Regs<N>::V) : "memory");
    // ======================= unpack V =======================
    // A lane takes 16 bytes (32 elements) of LOADS rows; eight neighbouring lanes are on four rows and two parts of a row: their
    // 16-byte stores fall on eight different bank groups.  Rows behind the last key are zeros.
    constexpr int LOADS = D / 32, STEP = TN / LOADS;
    const int u = warp - W_V;
    const int part = D == 128 ? (lane & 1) | ((lane >> 3) & 1) << 1 : lane & 1;
    const int row0 = (D == 128 ? u << 3 : u << 4) | (D == 128 ? ((lane >> 1) & 3) | (lane >> 4) << 2 : ((lane >> 1) & 3) | (lane >> 3) << 2);
    int at_rows[LOADS], at_scales[LOADS];  // where its rows and scales lie in the ring's tile
#pragma unroll
    for (int k = 0; k < LOADS; ++k) {
      const int key = row0 + k * STEP, slot = key & (M.P - 1), in_page = (key - slot) / M.P * 2 * slab + slab;
      at_rows[k] = in_page + slot * ROW + part * 16;
      at_scales[k] = in_page + M.P * ROW + slot * SC + part * 2;
    }
    bool ok = true;
    for (int i = 0; i < n_tiles && ok; ++i) {
      const int stage = i % V_STAGES, rs = i % RING;
      ok = __all_sync(0xffffffffu, wait_for(bar(B_RFULL + rs), (i / RING) & 1));
      const uint8_t* packed = smem + L::OFF_RING + rs * 2 * L::PACKED;
      const int valid = s_valid[rs];
      uint4 data[LOADS];
      uint32_t f[LOADS];
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        data[k] = *reinterpret_cast<const uint4*>(packed + at_rows[k]);
        f[k] = *reinterpret_cast<const uint16_t*>(packed + at_scales[k]);
        if (row0 + k * STEP >= valid) f[k] = 0;  // (zero times codes, which are finite)
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_REMPTY + rs));
      if (i >= V_STAGES && !__all_sync(0xffffffffu, wait_for(bar(B_VEMPTY + stage), (i / V_STAGES - 1) & 1))) ok = false;
      if (!ok) break;
      uint8_t* tile = smem + L::OFF_V + stage * V_BYTES + (part >> 1) * HALF_BYTES;
#pragma unroll
      for (int k = 0; k < LOADS; ++k) {
        const uint32_t w[4] = {data[k].x, data[k].y, data[k].z, data[k].w};
        const uint32_t f2 = e4m3_to_half2(f[k]), sc[2] = {low_twice(f2), high_twice(f2)};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const uint32_t h = sc[q >> 1];
          *reinterpret_cast<uint4*>(tile + swz128(row0 + k * STEP, (part & 1) * 4 + q)) =
              make_uint4(hmul2(e2m1_to_half2<0>(w[q]), h), hmul2(e2m1_to_half2<1>(w[q]), h), hmul2(e2m1_to_half2<2>(w[q]), h),
                         hmul2(e2m1_to_half2<3>(w[q]), h));
        }
      }
      fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_VFULL + stage));
    }
    if (!ok) timed_out(71, 0);
  } else if (warp < W_OTHER) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Regs<N>::SOFTMAX) : "memory");
    // ======================= softmax =======================
    const int group = (warp - W_SOFTMAX) >> 2, quad = warp & 3, me = quad * 32 + lane;  // the thread's key in the tile = its element of O
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    float* s_max = reinterpret_cast<float*>(smem + L::OFF_STATE + group * L::GROUP_STATE);  // [4][N]
    float* s_m = s_max + 4 * N;                                                              // [N] the rows' bases
    float* s_alpha = s_m + N;                                                                // [N] factors of O
    float2 m[N / 2];  // added to the scores: the rows' bases, negative, 0 for rows without a key
    float2 l[N / 2];  // sums over the thread's keys
    bool ok = true;
    int i = 0;  // tile of the run
    for (int pc = 0; at.left > 0 && ok; ++pc) {
      const int count = at.count(), buf = pc & 1;
      const int first_end = p.causal ? min(at.s.end, at.s.len + 1) : at.s.end;  // keys that the first row sees
      const uint32_t tO = tmem + lane_addr + TM_O + (2 * buf + group) * N;
      float mul = 0.f;
#pragma unroll
      for (int n = 0; n < N / 2; ++n) m[n] = l[n] = make_float2(0.f, 0.f);
      const int j0 = (i + group) & 1;  // the group's first tile of the piece
      // A wait runs out for a warp, not for its group: the loop is left at the group's votes alone, where all four warps agree, or a
      // warp would wait at one named barrier and the others at another.
      for (int j = j0; j < count; j += 2) {
        const int b = group, it = i + j, key = (at.tile + j) * TN + me;
        ok = ok & (bool)__all_sync(0xffffffffu, wait_for(bar(B_SFULL + b), (it >> 1) & 1));
        if (j == j0) mul = s_mul[pc & 3];  // (written before the MMAs that this barrier waits for)
        uint32_t v[N];
        tc_fence_after();
        tmem_ld_cols<N>(tmem + lane_addr + TM_S + b * N, v);
        tc_wait_ld();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_SFREE + b));
        float2 x[N / 2];
#pragma unroll
        for (int n = 0; n < N / 2; ++n) x[n] = make_float2(__uint_as_float(v[2 * n]), __uint_as_float(v[2 * n + 1]));
        if ((at.tile + j + 1) * TN > first_end) {  // (uniform for the tile)
          // token n / G sees the key if key <= len + n / G
          const int from = key >= at.s.end ? N : p.causal ? max(0, key - at.s.len) * M.G : 0;
#pragma unroll
          for (int n = 0; n < N; ++n)
            if (n < from) (n & 1 ? x[n / 2].y : x[n / 2].x) = -INFINITY;
        }
        const float2 mul2 = make_float2(mul, mul);
        float top = -INFINITY;
#pragma unroll
        for (int n = 0; n < N / 2; ++n) {
          const float2 e = __ffma2_rn(x[n], mul2, m[n]);
          top = max3(top, e.x, e.y);
        }
        if (softmax_any(group, j == j0 || top > kMostAboveBase || !ok)) {
          // a row's base moves (or the first tile sets it): the tile's over all its keys
          if (softmax_any(group, !ok)) {
            ok = false;
            break;
          }
#pragma unroll
          for (int n = 0; n < N; ++n) {
            const float c = warp_max(n & 1 ? x[n / 2].y : x[n / 2].x);
            if (lane == 0) s_max[quad * N + n] = base_of(c, mul);
          }
          softmax_sync(group);
          if (quad == 0 && lane < N) {
            const float c = fmaxf(fmaxf(s_max[lane], s_max[N + lane]), fmaxf(s_max[2 * N + lane], s_max[3 * N + lane]));
            const float old = j == j0 ? -INFINITY : s_m[lane];
            const bool grow = base_moves(c, old) || j == j0;
            s_alpha[lane] = grow ? (j == j0 || c == -INFINITY ? 1.f : fast_exp2(old - c)) : 1.f;
            s_m[lane] = grow ? c : old;
          }
          softmax_sync(group);
          if (j > j0) {
            ok = __all_sync(0xffffffffu, wait_for(bar(B_PEMPTY + b), ((it >> 1) - 1) & 1));  // O has the group's tile before
            tc_fence_after();
            uint32_t o[N];
            tmem_ld_cols<N>(tO, o);
            tc_wait_ld();
#pragma unroll
            for (int n = 0; n < N; ++n) {
              const float a = s_alpha[n];
              o[n] = __float_as_uint(__uint_as_float(o[n]) * a);
              (n & 1 ? l[n / 2].y : l[n / 2].x) *= a;
            }
            tmem_st_cols<N>(tO, o);
            tc_wait_st();
            tc_fence_before();
          }
#pragma unroll
          for (int n = 0; n < N / 2; ++n)
            m[n] = make_float2(s_m[2 * n] == -INFINITY ? 0.f : -s_m[2 * n], s_m[2 * n + 1] == -INFINITY ? 0.f : -s_m[2 * n + 1]);
        }
        uint32_t pk[N / 2];
#pragma unroll
        for (int n = 0; n < N / 2; ++n) {
          const float2 e = __ffma2_rn(x[n], mul2, m[n]), ex = make_float2(fast_exp2(e.x), fast_exp2(e.y));
          pk[n] = pack_half2(ex.x, ex.y);
          l[n] = __fadd2_rn(l[n], ex);
        }
        if (it >= 2) ok = ok & (bool)__all_sync(0xffffffffu, wait_for(bar(B_PEMPTY + b), ((it >> 1) - 1) & 1));
        uint8_t* prow = smem + L::OFF_P + b * P_BYTES;
#pragma unroll
        for (int q = 0; q < N / 8; ++q)
          *reinterpret_cast<uint4*>(prow + swz128(me, q)) = make_uint4(pk[4 * q], pk[4 * q + 1], pk[4 * q + 2], pk[4 * q + 3]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_PFULL + b));
      }
      // ---- the piece's end: the groups' sums meet ----
      if (ok) ok = __all_sync(0xffffffffu, wait_for(bar(B_OFULL + 2 * buf + group), (pc >> 1) & 1));
      // row sums over the warp's keys: lane n ends with row n's
      {
        float c[N];
#pragma unroll
        for (int n = 0; n < N / 2; ++n) c[2 * n] = l[n].x, c[2 * n + 1] = l[n].y;
        if constexpr (N == 16) {
#pragma unroll
          for (int n = 0; n < 16; ++n) c[n] += __shfl_xor_sync(0xffffffffu, c[n], 16);
        }
#pragma unroll
        for (int half = N / 2; half >= 1; half >>= 1) {
          const bool upper = lane & half;
#pragma unroll
          for (int n = 0; n < half; ++n) {
            const float give = upper ? c[n] : c[n + half], keep = upper ? c[n + half] : c[n];
            c[n] = keep + __shfl_xor_sync(0xffffffffu, give, half);
          }
        }
        if (lane < N) s_max[quad * N + lane] = c[0];
        if (j0 >= count && quad == 0 && lane < N) s_m[lane] = -INFINITY;  // (no tile of the piece)
      }
      tc_fence_after();
      uint32_t o[N];
      tmem_ld_cols<N>(tO, o);
      tc_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_OFREE + 2 * buf + group));
      if (j0 >= count) {
#pragma unroll
        for (int n = 0; n < N; ++n) o[n] = 0;
      }
      uint8_t* box = smem + L::OFF_P + P_BYTES;  // the second group's, whose products are done
      if (group == 1) {
#pragma unroll
        for (int q = 0; q < N / 4; ++q)
          *reinterpret_cast<uint4*>(box + swz128(me, q)) = make_uint4(o[4 * q], o[4 * q + 1], o[4 * q + 2], o[4 * q + 3]);
      }
      if (groups_any(!ok)) {
        ok = false;
        break;
      }
      const bool whole = at.tile == 0 && count == at.s.tiles;
      const int rows = at.s.n * M.G;
      const int64_t piece = 2 * (int64_t)blockIdx.x + (at.tile == 0);  // a run has one piece at most that starts before it, and one that ends behind it
      auto row_of = [&](int n) { return (int64_t)(at.s.t0 + n / M.G) * M.Hq + at.kh * M.G + n % M.G; };
      auto has_row = [&](int n) { return n < rows && (unsigned)at.s.t0 + (unsigned)(n / M.G) < (unsigned)p.total_q; };
      if (group == 0) {
        if (quad == 0 && lane < N) {
          const float* other = s_max + L::GROUP_STATE / 4;
          const float l0 = (s_max[lane] + s_max[N + lane]) + (s_max[2 * N + lane] + s_max[3 * N + lane]);
          const float l1 = (other[lane] + other[N + lane]) + (other[2 * N + lane] + other[3 * N + lane]);
          const float m0 = s_m[lane], m1 = other[4 * N + lane], top = fmaxf(m0, m1), least = top == -INFINITY ? 0.f : top;
          // (a group that saw no key of the row, or NaN alone, has no maximum: its sums, 0 or NaN, count as they are)
          const float f0 = m0 == -INFINITY ? 1.f : fast_exp2(m0 - least), f1 = m1 == -INFINITY ? 1.f : fast_exp2(m1 - least);
          const float sum = l0 * f0 + l1 * f1;
          const float out = whole ? (sum != 0.f ? p.v_scale / sum : 0.f) : p.v_scale;  // (a NaN among the inputs shows in the output)
          s_alpha[lane] = f0 * out;
          s_alpha[L::GROUP_STATE / 4 + lane] = f1 * out;
          if (has_row(lane)) {
            if (!whole) p.part_ml[piece * N + lane] = make_float2(top, sum);
            else if (p.lse) p.lse[row_of(lane)] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
          }
        }
        softmax_sync(0);
        if (me < D) {
          // row n's place in the output: the heads of a token follow one another
          int64_t to = whole ? ((int64_t)at.s.t0 * M.Hq + at.kh * M.G) * D + me : piece * N * D + me;
          const int left = min(rows, (int)min((int64_t)INT32_MAX, ((int64_t)p.total_q - at.s.t0) * M.G));  // rows with storage
          const int skip = whole ? (M.Hq - M.G) * D : 0;
          const bool fp32 = !whole || M.out_fp32;
          float* out32 = whole ? reinterpret_cast<float*>(p.out) : p.part_o;
          int h = 0;
#pragma unroll
          for (int q = 0; q < N / 4; ++q) {
            const float4 v = *reinterpret_cast<const float4*>(box + swz128(me, q));
            const float o1[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int n = 4 * q + e;
              const float y = __uint_as_float(o[n]) * s_alpha[n] + o1[e] * s_alpha[L::GROUP_STATE / 4 + n];
              if (n < left && to >= 0) {  // (a negative row offset has no storage either)
                if (fp32) out32[to] = y;
                else reinterpret_cast<__nv_bfloat16*>(p.out)[to] = __float2bfloat16(y);
              }
              to += D;
              if (++h == M.G) {
                h = 0;
                to += skip;
              }
            }
          }
        }
      }
      groups_any(false);  // (the second group's sums have been read)
      i += count;
      at.left -= count;
      at.tile += count;
      if (at.left > 0) at.next_stream(p);
    }
    if (!ok) timed_out(72, i);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Regs<N>::OTHER) : "memory");
    if (warp == W_OTHER) {
      // ======================= S = K Q^T =======================
      bool ok = true;
      int i = 0;
      for (int pc = 0; at.left > 0 && ok; ++pc) {
        const int count = at.count(), buf = pc & 1;
        ok = __all_sync(0xffffffffu, wait_for(bar(B_QFULL + buf), (pc >> 1) & 1));
        const uint64_t dq = smem_desc(sbase + L::OFF_Q + buf * L::Q_BYTES, 16);
        for (int j = 0; j < count && ok; ++j, ++i) {
          const int stage = i % K_STAGES, b = i & 1;
          ok = wait_for(bar(B_KFULL + stage), (i / K_STAGES) & 1);
          if (ok && i >= 2) ok = wait_for(bar(B_SFREE + b), ((i >> 1) - 1) & 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
              tc_mma_ts(tmem + TM_S + b * N, tmem + stage * K_COLS + ks * 8, desc_advance(dq, (ks >> 2) * N * 128 + (ks & 3) * 32), IDESC_S, ks > 0);
            tc_commit(bar(B_SFULL + b));
            tc_commit(bar(B_KEMPTY + stage));
            if (j + 1 == count) tc_commit(bar(B_QFREE + buf));
          }
          __syncwarp();
        }
        at.left -= count;
        at.tile += count;
        if (at.left > 0) at.next_stream(p);
      }
      if (!ok) timed_out(73, i);
    } else if (warp == W_OTHER + 1) {
      // ======================= O += V^T P^T =======================
      bool ok = true;
      int i = 0;
      const uint64_t dv0 = smem_desc(sbase + L::OFF_V, HALF_BYTES), dp0 = smem_desc(sbase + L::OFF_P, HALF_BYTES);
      for (int pc = 0; at.left > 0 && ok; ++pc) {
        const int count = at.count(), buf = pc & 1;
        if (pc >= 2)
          ok = __all_sync(0xffffffffu, wait_for(bar(B_OFREE + 2 * buf), ((pc >> 1) - 1) & 1) && wait_for(bar(B_OFREE + 2 * buf + 1), ((pc >> 1) - 1) & 1));
        for (int j = 0; j < count && ok; ++j, ++i) {
          const int stage = i % V_STAGES, b = i & 1;
          ok = wait_for(bar(B_VFULL + stage), (i / V_STAGES) & 1) && wait_for(bar(B_PFULL + b), (i >> 1) & 1);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t dv = desc_advance(dv0, stage * V_BYTES), dp = desc_advance(dp0, b * P_BYTES);
#pragma unroll
            for (int ks = 0; ks < TN / 16; ++ks)
              tc_mma_ss(tmem + TM_O + (2 * buf + b) * N, desc_advance(dv, ks * 2048), desc_advance(dp, ks * 2048), IDESC_O, j > 1 || ks > 0);
            tc_commit(bar(B_VEMPTY + stage));
            tc_commit(bar(B_PEMPTY + b));
            if (j + 1 == count) {
              tc_commit(bar(B_OFULL + 2 * buf));
              tc_commit(bar(B_OFULL + 2 * buf + 1));
            }
          }
          __syncwarp();
        }
        at.left -= count;
        at.tile += count;
        if (at.left > 0) at.next_stream(p);
      }
      if (!ok) timed_out(74, i);
    } else if (warp == W_OTHER + 2) {
      // ======================= Q =======================
      // Lane n brings row n to fp16, in the order of K's elements.  All rows of a stream are multiplied by the same power of two,
      // which brings the largest element of them all to [2^14, 2^15).
      bool ok = true;
      for (int pc = 0; at.left > 0 && ok; ++pc) {
        const int count = at.count(), buf = pc & 1;
        if (pc >= 2) ok = __all_sync(0xffffffffu, wait_for(bar(B_QFREE + buf), ((pc >> 1) - 1) & 1));
        if (!ok) break;
        const int n = lane & (N - 1), tok = n / M.G;
        const bool there = n < at.s.n * M.G && (unsigned)at.s.t0 + (unsigned)tok < (unsigned)p.total_q;
        const __nv_bfloat16* row = p.q + ((int64_t)(at.s.t0 + tok) * M.Hq + at.kh * M.G + n % M.G) * D;
        float amax = 0.f;
#pragma unroll 4
        for (int k = 0; k < D / 8; ++k) {
          const uint4 v = there ? *reinterpret_cast<const uint4*>(row + 8 * k) : make_uint4(0, 0, 0, 0);
          const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 y = unpack_bf16x2(u[e]);
            amax = finite_max(amax, y);
          }
        }
#pragma unroll
        for (int sh = 16; sh >= 1; sh >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, sh));
        float up, down;
        q_powers(amax, &up, &down);
        uint8_t* to = smem + L::OFF_Q + buf * L::Q_BYTES;
        // chunk ch of eight: elements D / 4 t + 4 j + 0 .. 3 of t = 2 (ch & 1) and of the t behind, j = ch / 2
#pragma unroll 4
        for (int ch = 0; ch < D / 8; ++ch) {
          uint32_t o[4];
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint2 v = there ? *reinterpret_cast<const uint2*>(row + D / 4 * (2 * (ch & 1) + x) + 4 * (ch >> 1)) : make_uint2(0, 0);
            const float2 a = unpack_bf16x2(v.x), c = unpack_bf16x2(v.y);
            o[2 * x] = pack_half2(a.x * up, a.y * up);
            o[2 * x + 1] = pack_half2(c.x * up, c.y * up);
          }
          if (lane < N) *reinterpret_cast<uint4*>(to + (ch >> 3) * N * 128 + swz128(n, ch & 7)) = make_uint4(o[0], o[1], o[2], o[3]);
        }
        if (lane == 0) s_mul[pc & 3] = fmaxf(down * p.scale_log2, 0x1p-126f);  // (never 0: a masked score stays minus infinity)
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_QFULL + buf));
        at.left -= count;
        at.tile += count;
        if (at.left > 0) at.next_stream(p);
      }
      if (!ok) timed_out(75, 0);
    } else {
      // ======================= pages =======================
      // Two tiles at a time (a wait for the ring costs some hundred cycles, and these overlap), a lane per page; the page ids of the two
      // tiles behind are on their way meanwhile.  One TMA load brings K and V of a page: each load's issue takes the warp some hundred
      // cycles, too.
      const int page_shift = 31 - __clz(M.P), ppt = TN >> page_shift;  // pages per tile: 2, 4 or 8
      const int sub = lane & (ppt - 1), ahead = lane / ppt;            // (idle lanes: ahead > 1)
      bool ok = true;
      // the lane's tile of the two: its request, KV head, keys, pages and the page id
      int t_r = 0, t_kh = 0, t_valid = 0, t_here = 0, t_place = 0, t_page = 0;
      bool t_mine = false;
      auto take = [&]() {
        t_mine = false;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (at.left == 0) break;
          if (k == ahead) {
            t_mine = true;
            t_r = at.r;
            t_kh = at.kh;
            t_valid = min(TN, at.s.end - at.tile * TN);
            t_here = max(0, min(ppt, (t_valid + M.P - 1) >> page_shift));
            t_place = at.tile * ppt + sub;
            t_page = sub < t_here ? p.b.block_table[(int64_t)at.r * p.b.max_blocks + t_place] : 0;
          }
          --at.left;
          if (++at.tile == at.s.tiles && at.left > 0) at.next_stream(p);
        }
      };
      if (lane == 0) tma_prefetch_desc(&tm_pool);
      take();
      int rs = ahead % RING, round = 0;  // the lane's slot of the ring, and how often it has been around
      for (int i = 0; i < n_tiles; i += 2) {
        const bool mine = t_mine;
        const int r = t_r, kh = t_kh, valid = t_valid, here = t_here, place = t_place;
        int page = t_page;
        take();
        if (mine && sub < here && (page < 0 || page >= p.num_pages)) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, place, page);
          page = 0;
        }
        if (mine && round > 0) ok = wait_for(bar(B_REMPTY + rs), (round - 1) & 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (mine && sub == 0) {
          s_valid[rs] = valid;
          mbar_arrive_expect_tx(bar(B_RFULL + rs), 2 * here * slab);
        }
        __syncwarp();
        if (mine && sub < here)
          tma_load_5d(sbase + L::OFF_RING + rs * 2 * L::PACKED + sub * 2 * slab, &tm_pool, bar(B_RFULL + rs), 0, 0, kh, 0, page);
        rs += 2;
        if (rs >= RING) {
          rs -= RING;
          ++round;
        }
      }
      if (!ok) timed_out(76, 0);
    }
  }

  // ---- teardown: everyone is done with TMEM before it is released ----
  tc_fence_before();
  __syncthreads();
  if (warp == W_OTHER) {
    if (*reinterpret_cast<const volatile int32_t*>(p.err) == HSWA_ERR_TIMEOUT) __nanosleep(100000);  // (MMAs in flight that nobody waited for)
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TM_COLS) : "memory");
  }
}

template <int D, int N>
cudaError_t launch(const CUtensorMap& tm_pool, const PackedAttnParams& p, cudaStream_t s) {
  auto kern = packed_rows_kernel<D, N>;
  cudaError_t e = hswa_prepare_kernel<packed_rows_kernel<D, N>>(Smem<D, N>::BYTES);
  if (e != cudaSuccess) return e;
  // the softmax warps' request for registers is granted only if the launch gives the block 640 x 96
  static const cudaError_t budget = [&] {
    cudaFuncAttributes attr;
    const cudaError_t q = cudaFuncGetAttributes(&attr, kern);
    return q != cudaSuccess ? q : attr.numRegs < 96 ? cudaErrorLaunchOutOfResources : cudaSuccess;
  }();
  if (budget != cudaSuccess) return budget;
  kern<<<p.runs, kThreads, Smem<D, N>::BYTES, s>>>(tm_pool, p);
  e = cudaGetLastError();
  return e != cudaSuccess ? e : hswa_launch_packed_join(p, N, TN, s);
}

}  // namespace

cudaError_t hswa_launch_packed_rows(const CUtensorMap& tm_pool, const PackedAttnParams& p, int rows, cudaStream_t s) {
  if (p.m.D == 128) return rows <= 16 ? launch<128, 16>(tm_pool, p, s) : launch<128, 32>(tm_pool, p, s);
  return rows <= 16 ? launch<64, 16>(tm_pool, p, s) : launch<64, 32>(tm_pool, p, s);
}
