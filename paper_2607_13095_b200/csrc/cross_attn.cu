// Cross attention to an encoder's states, held in the pages of a Full layer (paper Sec. 3.1.1: one logical view over
// paged storage): softmax(scale q K^T) V over all len_r cached positions of the request, no causal mask, any number of
// query tokens per request; a request without states gives zeros and a log-sum-exp of minus infinity.  Single tokens run
// on the streaming decode kernel, everything else on the tcgen05 tile kernel; here is the join of its key slices.
#include "hswa_internal.cuh"

namespace {
using namespace hswa_dev;

// Joins the key slices: out = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.  One warp per (token, head); slices that hold
// no key of the row (l = 0) are passed over.
template <int D>
__global__ void __launch_bounds__(128) cross_combine_kernel(const CrossParams p) {
  const int64_t row = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  const ModelParams& M = p.m;
  // launched early (programmatic dependent launch) behind the kernel that writes the partials
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (row >= (int64_t)(p.q_end ? min(*p.q_end, p.total_q) : p.total_q) * M.Hq) return;
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

}  // namespace

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
