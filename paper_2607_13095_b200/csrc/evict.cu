// Eviction from a Full layer's cache by accumulated attention weight: the choice of the positions that stay, and their move
// to the head of fresh pages (paper Sec. 3.1.3: pages may be shared between
// requests, so kept rows are copied to pages of the request's own, never moved inside pages that another one reads).
#include "hswa_internal.cuh"

namespace {
using namespace hswa_dev;

// ---------------------------------------------------------------------------------------------------------------------
// Order-preserving map of a weight to 32 bits: NaN lowest, -0 and +0 alike, protected positions above everything.
__device__ __forceinline__ uint32_t rank_key(float w, int j, int ctx, int first, int last) {
  if (j < first || j >= ctx - last) return 0xffffffffu;
  if (w != w) return 0u;
  if (w == 0.f) return 0x80000000u;
  const uint32_t u = __float_as_uint(w);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// One block per (request, KV head): the keep-th largest key by four passes over 8-bit digits, then the kept positions in
// ascending order, ties taken from the lowest index on.
constexpr int ST = 1024;
__global__ void __launch_bounds__(ST) evict_select_kernel(const SelectParams p) {
  __shared__ int hist[256];
  __shared__ uint32_t s_prefix;
  __shared__ int s_want;
  __shared__ int warp_gt[ST / 32], warp_eq[ST / 32];
  const int kh = blockIdx.x % p.Hkv, r = blockIdx.x / p.Hkv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int ctx = p.ctx_len[r];
  int keep = p.keep_len[r];
  if (ctx < 0 || ctx > p.max_ctx_len || keep < 0 || keep > p.max_keep) {
    if (tid == 0 && kh == 0)
      record_error(p.err, HSWA_ERR_BOUNDS, r, ctx < 0 || ctx > p.max_ctx_len ? -1 : -2, ctx < 0 || ctx > p.max_ctx_len ? ctx : keep);
    ctx = max(0, min(ctx, p.max_ctx_len));
    keep = max(0, min(keep, p.max_keep));
  }
  keep = min(keep, ctx);
  const float* w = p.weights + ((int64_t)r * p.Hkv + kh) * p.stride;
  int32_t* out = p.keep_idx + ((int64_t)r * p.Hkv + kh) * p.max_keep;
  if (tid == 0 && kh == 0) p.kept_len[r] = keep;
  for (int i = keep + tid; i < p.max_keep; i += ST) out[i] = -1;
  if (keep == 0) return;
  if (tid == 0) {
    s_prefix = 0;
    s_want = keep;
  }
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += ST) hist[i] = 0;
    __syncthreads();
    const uint32_t prefix = s_prefix;
    for (int j = tid; j < ctx; j += ST) {
      const uint32_t k = rank_key(w[j], j, ctx, p.protect_first, p.protect_last);
      if (shift == 24 || (k >> (shift + 8)) == prefix) atomicAdd(&hist[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {
      int want = s_want, d = 255;
      while (want > hist[d]) want -= hist[d--];
      s_want = want;
      s_prefix = (prefix << 8) | (uint32_t)d;
    }
    __syncthreads();
  }
  const uint32_t thr = s_prefix;
  const int ties = s_want;  // positions with exactly the threshold that stay
  int gt_base = 0, eq_base = 0;
  for (int j0 = 0; j0 < ctx; j0 += ST) {
    const int j = j0 + tid;
    const uint32_t k = j < ctx ? rank_key(w[j], j, ctx, p.protect_first, p.protect_last) : 0u;
    const unsigned gt = __ballot_sync(0xffffffffu, j < ctx && k > thr), eq = __ballot_sync(0xffffffffu, j < ctx && k == thr);
    if (lane == 0) {
      warp_gt[warp] = __popc(gt);
      warp_eq[warp] = __popc(eq);
    }
    __syncthreads();
    int g = gt_base, e = eq_base, gt_all = 0, eq_all = 0;
    for (int i = 0; i < ST / 32; ++i) {
      if (i < warp) {
        g += warp_gt[i];
        e += warp_eq[i];
      }
      gt_all += warp_gt[i];
      eq_all += warp_eq[i];
    }
    const unsigned below = (1u << lane) - 1;
    const int gr = g + __popc(gt & below), er = e + __popc(eq & below);
    const bool is_gt = (gt >> lane) & 1u, is_eq = (eq >> lane) & 1u;
    if (is_gt || (is_eq && er < ties)) out[gr + min(er, ties)] = j;
    gt_base += gt_all;
    eq_base += eq_all;
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Kept row i of (request, KV head) goes from the storage of position keep_idx[i] to that of position i behind the new
// block table.  One warp per kept row, K and V.
__global__ void __launch_bounds__(256) evict_compact_kernel(const CompactParams p) {
  const ModelParams& M = p.m;
  const int kh = blockIdx.y, r = blockIdx.z, lane = threadIdx.x & 31;
  const int i = blockIdx.x * 8 + (threadIdx.x >> 5);
  int kept = p.kept_len[r];
  const int ctx = min(p.b.ctx_len[r], p.max_ctx_len);
  if (kept < 0 || kept > p.max_keep) {
    if (threadIdx.x == 0 && blockIdx.x == 0 && kh == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, kept);
    kept = min(kept, p.max_keep);
  }
  if (i >= kept) return;
  const int64_t pair = (int64_t)r * M.Hkv + kh;
  const int j = p.keep_idx[pair * p.max_keep + i];
  if (j < 0 || j >= ctx) {
    if (lane == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, i, j);
    return;
  }
  const int src = p.b.block_table[(int64_t)r * p.b.max_blocks + j / M.P];
  const int dst = p.dst_block_table[(int64_t)r * p.dst_max_blocks + i / M.P];
  if (src < 0 || src >= p.num_pages || dst < 0 || dst >= p.num_pages) {
    if (lane == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, i, src < 0 || src >= p.num_pages ? src : dst);
    return;
  }
  const int chunks = M.D / 8;
  for (int c = lane; c < 2 * chunks; c += 32) {
    const int kv = c / chunks, ch = c % chunks;
    const uint4 v = *reinterpret_cast<const uint4*>(p.pool + ((((int64_t)src * 2 + kv) * M.Hkv + kh) * M.P + j % M.P) * M.D + ch * 8);
    *reinterpret_cast<uint4*>(p.pool + ((((int64_t)dst * 2 + kv) * M.Hkv + kh) * M.P + i % M.P) * M.D + ch * 8) = v;
  }
  if (p.weights && lane == 0) p.weights_out[pair * p.out_stride + i] = p.weights[pair * p.stride + j];
}

}  // namespace

cudaError_t hswa_launch_evict_select(const SelectParams& p, cudaStream_t s) {
  if (p.B == 0) return cudaSuccess;
  evict_select_kernel<<<p.B * p.Hkv, ST, 0, s>>>(p);
  return cudaGetLastError();
}

cudaError_t hswa_launch_evict_compact(const CompactParams& p, cudaStream_t s) {
  if (p.b.B == 0 || p.max_keep == 0) return cudaSuccess;
  dim3 grid((p.max_keep + 7) / 8, p.m.Hkv, p.b.B);
  evict_compact_kernel<<<grid, 256, 0, s>>>(p);
  return cudaGetLastError();
}
