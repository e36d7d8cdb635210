// Cross attention to an encoder's states, held in the pages of a Full layer (paper Sec. 3.1.1: one logical view over
// paged storage): softmax(scale q K^T) V over all len_r cached positions of the request, no causal mask, any number of
// query tokens per request; a request without states gives zeros and a log-sum-exp of minus infinity.  Single tokens run
// on the streaming decode kernel, everything else on the tcgen05 tile kernel; here is the join of its key slices.
#include "hswa_internal.cuh"

namespace {
using namespace hswa_dev;

// Joins the key slices: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  One warp per (token, head); slices that hold
// no key of the row (l = 0) are passed over, and a row that no block computed (past max_q_len: l < 0 in its first slice)
// stays as it was.  WPR = 4: four warps per row, a block's, each with every fourth slice, for more than eight of them: one
// warp pays a memory latency for every few (8 tokens against 32000 states, 32 / 8 heads of 128, 36 slices: 42 us, with four
// warps 34).
template <int D, int WPR>
__global__ void __launch_bounds__(128) cross_combine_kernel(const CrossParams p) {
  const int64_t row = WPR == 4 ? (int64_t)blockIdx.x : ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int sub = WPR == 4 ? (int)(threadIdx.x >> 5) : 0;
  const int lane = threadIdx.x & 31;
  const ModelParams& M = p.m;
  // launched early (programmatic dependent launch) behind the kernel that writes the partials
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (row < (int64_t)p.q_indptr[0] * M.Hq || row >= (int64_t)min(p.q_indptr[p.batch], p.total_q) * M.Hq) return;
  const float2* ml = p.part_ml + row * p.slices;
  const float* po = p.part_o + row * p.slices * D;
  float mm = -INFINITY;
  bool no_block = false;
  for (int s = lane; s < p.slices; s += 32) {
    const float2 v = ml[s];
    if (v.y != 0.f) mm = fmaxf(mm, v.x);
    no_block |= v.y < 0.f;
  }
  if (__any_sync(0xffffffffu, no_block)) return;
#pragma unroll
  for (int sh = 16; sh >= 1; sh >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, sh));
  constexpr int PER = D / 32;
  float acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.f;
  float L = 0.f;
  for (int s = sub; s < p.slices; s += WPR) {
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
  if constexpr (WPR == 4) {
    __shared__ float sums[3][32][PER + 1];
    if (sub > 0) {
#pragma unroll
      for (int i = 0; i < PER; ++i) sums[sub - 1][lane][i] = acc[i];
      sums[sub - 1][lane][PER] = L;
    }
    __syncthreads();
    if (sub > 0) return;
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
      for (int i = 0; i < PER; ++i) acc[i] += sums[k][lane][i];
      L += sums[k][lane][PER];
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

}  // namespace

cudaError_t hswa_launch_cross_combine(const CrossParams& p, cudaStream_t s) {
  const bool four = p.slices > 8;  // warps per row
  const int64_t rows = (int64_t)p.total_q * p.m.Hq, blocks = four ? rows : (rows + 3) / 4;
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
  if (four)
    return p.m.D == 128 ? cudaLaunchKernelEx(&cfg, cross_combine_kernel<128, 4>, p) : cudaLaunchKernelEx(&cfg, cross_combine_kernel<64, 4>, p);
  return p.m.D == 128 ? cudaLaunchKernelEx(&cfg, cross_combine_kernel<128, 1>, p) : cudaLaunchKernelEx(&cfg, cross_combine_kernel<64, 1>, p);
}
