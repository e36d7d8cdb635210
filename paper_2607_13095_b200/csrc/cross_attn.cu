// Cross attention to an encoder's states, held in the pages of a Full layer (paper Sec. 3.1.1: one logical view over
// paged storage): softmax(scale q K^T) V over all len_r cached positions of the request, no causal mask, any number of
// query tokens per request; a request without states gives zeros and a log-sum-exp of minus infinity.
//
// Tile kernel on warp-level tensor-core MMA for head_dim 64 (head_dim 128 takes the tcgen05 tile kernel, single tokens the
// streaming decode kernel).  No mask depends on the query, so the (token, head) rows of a GQA group are interchangeable: a block takes 64 packed rows of one (request, KV head) -- 8
// tokens at a group of 8 -- and the whole group shares each K/V tile.  Few rows against many keys do not fill the
// machine by themselves: the keys are then cut into slices whose (m, l, o) partials a second kernel joins.
#include "hswa_internal.cuh"

namespace {
using namespace hswa_dev;

constexpr int BM = 64;  // packed rows per block
constexpr int BN = 64;  // keys per tile

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void* src, bool pred) {
  const int sz = pred ? 16 : 0;  // size 0 zero-fills the destination
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(sz) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int D>
__global__ void __launch_bounds__(128, 2) cross_mma_kernel(const CrossParams p) {
  constexpr int HALF_BYTES = BN * 128;
  constexpr int TILE_BYTES = (D / 64) * HALF_BYTES;  // one K or V or Q tile
  constexpr int CHUNKS = D / 8;
  constexpr int KS = D / 16;
  constexpr int NT_O = D / 8;

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  const uint32_t sQ = smem_u32(smem);
  const uint32_t sKV = sQ + TILE_BYTES;  // [2 buffers][K, V][TILE_BYTES]

  const ModelParams& M = p.m;
  unsigned item = blockIdx.x;
  const int rt = item % p.row_tiles;
  item /= p.row_tiles;
  const int slice = item % p.slices;
  item /= p.slices;
  const int kh = item % M.Hkv, r = item / M.Hkv;
  const int t0 = p.b.q_indptr ? p.b.q_indptr[r] : r;
  const int n = p.b.q_indptr ? p.b.q_indptr[r + 1] - t0 : 1;
  const int row0 = rt * BM;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ctx = p.b.ctx_len[r];
  if (tid == 0 && rt == 0 && slice == 0 && kh == 0) {  // the grid was sized from the host's bounds
    if (ctx < 0 || ctx > p.max_ctx_len) record_error(p.err, HSWA_ERR_BOUNDS, r, -1, ctx);
    if (n < 0 || n > p.max_q_len) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, n);
  }
  const int rows = min(BM, n * M.G - row0);
  if (rows <= 0) return;
  const int k_begin = slice * p.slice_len;
  const int k_end = min(min(ctx, p.max_ctx_len), k_begin + p.slice_len);
  const int n_tiles = k_end > k_begin ? (k_end - k_begin + BN - 1) / BN : 0;

  auto q_row = [&](int row) { return (int64_t)(t0 + (row0 + row) / M.G) * M.Hq + kh * M.G + (row0 + row) % M.G; };

  // ---- Q tile -> shared (rows past the request's end are zero) ----
  for (int idx = tid; idx < BM * CHUNKS; idx += 128) {
    const int row = idx / CHUNKS, ch = idx % CHUNKS;
    const bool ok = row < rows;
    cp_async_16(sQ + (ch >> 3) * HALF_BYTES + swz128(row, ch & 7), p.q + q_row(ok ? row : 0) * D + ch * 8, ok);
  }
  cp_async_commit();

  // positions at or past k_end (a page's tail may hold anything) and bad pages are zero-filled: 0 x NaN never happens
  auto load_kv = [&](int tile, int buf) {
    const int j0 = k_begin + tile * BN;
    const uint32_t sK = sKV + buf * 2 * TILE_BYTES, sV = sK + TILE_BYTES;
    for (int idx = tid; idx < BN * CHUNKS; idx += 128) {
      const int row = idx / CHUNKS, ch = idx % CHUNKS;
      const int j = j0 + row;
      const __nv_bfloat16 *ks = p.pool, *vs = p.pool;
      bool ok = j < k_end;
      if (ok) {
        const int page = p.b.block_table[(int64_t)r * p.b.max_blocks + j / M.P];
        if (page < 0 || page >= p.num_pages) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, j / M.P, page);
          ok = false;
        } else {
          ks = p.pool + ((((int64_t)page * 2 + 0) * M.Hkv + kh) * M.P + j % M.P) * D + ch * 8;
          vs = ks + (int64_t)M.Hkv * M.P * D;
        }
      }
      const uint32_t o = (ch >> 3) * HALF_BYTES + swz128(row, ch & 7);
      cp_async_16(sK + o, ks, ok);
      cp_async_16(sV + o, vs, ok);
    }
    cp_async_commit();
  };

  if (n_tiles > 0) load_kv(0, 0);

  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
  float o[NT_O][4];
#pragma unroll
  for (int i = 0; i < NT_O; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  uint32_t qf[KS][4];
  const int mi = lane >> 3, mr = lane & 7;

  for (int tile = 0; tile < n_tiles; ++tile) {
    const int buf = tile & 1;
    if (tile + 1 < n_tiles) {
      load_kv(tile + 1, buf ^ 1);
      cp_async_wait<1>();
    } else {
      cp_async_wait<0>();
    }
    __syncthreads();
    if (tile == 0) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int row = warp * 16 + (mi & 1) * 8 + mr;
        const int chunk = 2 * ks + (mi >> 1);
        ldmatrix_x4(sQ + (chunk >> 3) * HALF_BYTES + swz128(row, chunk & 7), qf[ks][0], qf[ks][1], qf[ks][2], qf[ks][3]);
      }
    }
    const uint32_t sK = sKV + buf * 2 * TILE_BYTES, sV = sK + TILE_BYTES;

    float s[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll
    for (int np = 0; np < 4; ++np) {
      const int key = np * 16 + (mi >> 1) * 8 + mr;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const int chunk = 2 * ks + (mi & 1);
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4(sK + (chunk >> 3) * HALF_BYTES + swz128(key, chunk & 7), b0, b1, b2, b3);
        mma_bf16_16816(s[2 * np], qf[ks][0], qf[ks][1], qf[ks][2], qf[ks][3], b0, b1);
        mma_bf16_16816(s[2 * np + 1], qf[ks][0], qf[ks][1], qf[ks][2], qf[ks][3], b2, b3);
      }
    }
    const int live = k_end - (k_begin + tile * BN);  // keys of this tile, for every row alike
    float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int key = nt * 8 + (lane & 3) * 2 + (e & 1);
        const float v = key < live ? s[nt][e] * M.scale_log2 : -INFINITY;
        s[nt][e] = v;
        mx[e >> 1] = fmaxf(mx[e >> 1], v);
      }
    }
    float m_use[2], alpha[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 1));
      mx[j] = fmaxf(mx[j], __shfl_xor_sync(0xffffffffu, mx[j], 2));
      const float m_new = fmaxf(m_run[j], mx[j]);
      m_use[j] = m_new == -INFINITY ? 0.f : m_new;
      alpha[j] = fast_exp2(m_run[j] - m_use[j]);
      m_run[j] = m_new;
      l_run[j] *= alpha[j];
    }
#pragma unroll
    for (int i = 0; i < NT_O; ++i) {
      o[i][0] *= alpha[0];
      o[i][1] *= alpha[0];
      o[i][2] *= alpha[1];
      o[i][3] *= alpha[1];
    }
    // the row sums take the fp32 values before their rounding to bf16: the log-sum-exp is a result that
    // hswa_attn_weights exponentiates again
    uint32_t pa[4][4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int nt = 2 * kk + half;
        const float e0 = fast_exp2(s[nt][0] - m_use[0]), e1 = fast_exp2(s[nt][1] - m_use[0]);
        const float e2 = fast_exp2(s[nt][2] - m_use[1]), e3 = fast_exp2(s[nt][3] - m_use[1]);
        l_run[0] += e0 + e1;
        l_run[1] += e2 + e3;
        pa[kk][half * 2 + 0] = pack_bf16x2(e0, e1);
        pa[kk][half * 2 + 1] = pack_bf16x2(e2, e3);
      }
    }
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) {
      const int key = kk * 16 + (mi & 1) * 8 + mr;
#pragma unroll
      for (int dp = 0; dp < D / 16; ++dp) {
        const int chunk = 2 * dp + (mi >> 1);
        uint32_t b0, b1, b2, b3;
        ldmatrix_x4_trans(sV + (chunk >> 3) * HALF_BYTES + swz128(key, chunk & 7), b0, b1, b2, b3);
        mma_bf16_16816(o[2 * dp], pa[kk][0], pa[kk][1], pa[kk][2], pa[kk][3], b0, b1);
        mma_bf16_16816(o[2 * dp + 1], pa[kk][0], pa[kk][1], pa[kk][2], pa[kk][3], b2, b3);
      }
    }
    __syncthreads();
  }
  cp_async_wait<0>();  // a slice without keys leaves with its Q load landed

  // ---- epilogue ----
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    l_run[j] += __shfl_xor_sync(0xffffffffu, l_run[j], 1);
    l_run[j] += __shfl_xor_sync(0xffffffffu, l_run[j], 2);
  }
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int row = warp * 16 + (lane >> 2) + half * 8;
    if (row >= rows) continue;
    const float L = l_run[half];
    const int64_t orow = q_row(row);
    if (p.slices > 1) {
      float* dst = p.part_o + (orow * p.slices + slice) * D;
#pragma unroll
      for (int nt = 0; nt < NT_O; ++nt)
        *reinterpret_cast<float2*>(dst + nt * 8 + (lane & 3) * 2) = make_float2(o[nt][half * 2], o[nt][half * 2 + 1]);
      if ((lane & 3) == 0) p.part_ml[orow * p.slices + slice] = make_float2(m_run[half], L);
      continue;
    }
    const float inv = L != 0.f ? 1.f / L : 0.f;  // (a NaN among the inputs shows in the output)
#pragma unroll
    for (int nt = 0; nt < NT_O; ++nt) {
      const int d = nt * 8 + (lane & 3) * 2;
      const float x = o[nt][half * 2] * inv, y = o[nt][half * 2 + 1] * inv;
      if (M.out_fp32)
        *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + orow * D + d) = make_float2(x, y);
      else
        *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(p.out) + orow * D + d) =
            __floats2bfloat162_rn(x, y);
    }
    if ((lane & 3) == 0 && p.lse)
      p.lse[orow] = L != 0.f ? (m_run[half] + log2f(L)) * 0.6931471805599453f : -INFINITY;
  }
}

// Joins the key slices: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  One warp per (token, head); slices that hold
// no key of the row (l = 0) are passed over.
template <int D>
__global__ void __launch_bounds__(128) cross_combine_kernel(const CrossParams p) {
  const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  const ModelParams& M = p.m;
  // launched early (programmatic dependent launch) behind the kernel that writes the partials
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (row >= (int64_t)p.total_q * M.Hq) return;
  const float2* ml = p.part_ml + row * p.slices;
  const float* po = p.part_o + row * p.slices * D;
  float mm = -INFINITY;
  for (int s = lane; s < p.slices; s += 32) {
    const float2 v = ml[s];
    if (v.y != 0.f) mm = fmaxf(mm, v.x);
  }
#pragma unroll
  for (int sh = 16; sh >= 1; sh >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, sh));
  constexpr int PER = D / 32;
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  float L = 0.f;
  for (int s = 0; s < p.slices; ++s) {
    const float2 v = ml[s];
    if (v.y == 0.f) continue;
    const float f = fast_exp2(v.x - mm);
    L += f * v.y;
#pragma unroll
    for (int i = 0; i < PER; i += 2) {
      const float2 x = *reinterpret_cast<const float2*>(po + (int64_t)s * D + lane * PER + i);
      acc[i] += f * x.x;
      acc[i + 1] += f * x.y;
    }
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;  // (a NaN among the inputs shows in the output)
#pragma unroll
  for (int i = 0; i < PER; i += 2) {
    const int64_t at = row * D + lane * PER + i;
    if (M.out_fp32)
      *reinterpret_cast<float2*>(reinterpret_cast<float*>(p.out) + at) = make_float2(acc[i] * inv, acc[i + 1] * inv);
    else
      *reinterpret_cast<__nv_bfloat162*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at) =
          __floats2bfloat162_rn(acc[i] * inv, acc[i + 1] * inv);
  }
  if (lane == 0 && p.lse) p.lse[row] = L != 0.f ? (mm + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

template <int D>
cudaError_t launch_mma_t(const CrossParams& p, cudaStream_t s) {
  constexpr int SMEM = 5 * (D / 64) * BN * 128 + 1024;
  auto kern = cross_mma_kernel<D>;
  cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (int64_t)p.row_tiles * p.slices * p.m.Hkv * p.b.B;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  kern<<<(unsigned)blocks, 128, SMEM, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

int hswa_cross_mma_rows() { return BM; }

cudaError_t hswa_launch_cross_mma(const CrossParams& p, cudaStream_t s) {
  if (p.m.D == 64) return launch_mma_t<64>(p, s);
  return cudaErrorInvalidValue;
}

cudaError_t hswa_launch_cross_combine(const CrossParams& p, cudaStream_t s) {
  const int64_t blocks = ((int64_t)p.total_q * p.m.Hq * 32 + 127) / 128;
  if (blocks > INT32_MAX) return cudaErrorInvalidConfiguration;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks, 1, 1);
  cfg.blockDim = dim3(128, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return p.m.D == 128 ? cudaLaunchKernelEx(&cfg, cross_combine_kernel<128>, p) : cudaLaunchKernelEx(&cfg, cross_combine_kernel<64>, p);
}
