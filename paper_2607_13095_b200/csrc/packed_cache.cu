// Rows into and out of a 4-bit cache (hswa_packed_append, hswa_packed_read): one thread per block of 16 elements.
//
// A block of 16 elements x with largest magnitude a, in a layer of scale g, is held as f = e4m3((a / g) / 6), s = f g, and
// e2m1(x / s): both roundings to the nearest, ties to the even code, at most 448 and 6.  x / s lies halfway between two levels
// often (both have few bits), so the quotient has to be right to the last bit: a product with 1 / s, then one Newton step on
// its exact residual.
// Bound by HBM: 2 bytes per element read, 0.5625 written (read-back: the reverse).
#include "packed.cuh"

namespace {
using namespace hswa_dev;

constexpr int kThreads = 256;

struct RowAt {
  int64_t slab;  // byte offset of the row's slab for K; V is Hkv slabs further on
  int slot;
  bool ok;
};

// Where the row of token `tok` (of all requests' tokens) is held; records what is out of range.
__device__ __forceinline__ RowAt find_row(const PackedCacheParams& p, int tok, int kh) {
  const ModelParams& M = p.m;
  RowAt at = {0, 0, false};
  int r = tok, i = 0;
  if (p.b.q_indptr) {
    if (tok < p.b.q_indptr[0]) return at;
    int lo = 0, hi = p.b.B;  // q_indptr[lo] <= tok, and tok < q_indptr[hi] unless hi = B
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.b.q_indptr[mid] <= tok) lo = mid; else hi = mid;
    }
    r = lo;
    i = tok - p.b.q_indptr[r];
    const int n = p.b.q_indptr[r + 1] - p.b.q_indptr[r];
    if (i >= n) return at;  // behind the last request
    if (n > p.max_q_len) {
      if (i == p.max_q_len) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, n);
      if (i >= p.max_q_len) return at;
    }
  }
  const int ctx = p.b.ctx_len[r];
  if (ctx < 0 || ctx > p.max_ctx_len) {
    record_error(p.err, HSWA_ERR_BOUNDS, r, -1, ctx);
    return at;
  }
  const int pos = ctx + i, block = pos / M.P;
  if (block >= p.b.max_blocks) {
    record_error(p.err, HSWA_ERR_BOUNDS, r, block, -1);
    return at;
  }
  const int page = p.b.block_table[(int64_t)r * p.b.max_blocks + block];
  if (page < 0 || page >= p.num_pages) {
    record_error(p.err, HSWA_ERR_BOUNDS, r, block, page);
    return at;
  }
  const int slab = M.P * (M.D / 2 + M.D / 16);
  at.slab = ((int64_t)page * 2 * M.Hkv + kh) * slab;
  at.slot = pos - block * M.P;
  at.ok = true;
  return at;
}

// Block number `it` of all tokens' rows: the 16 elements it % (D / 16) of KV head and token.
struct Item {
  int tok, kh, blk;
};
__device__ __forceinline__ Item item_of(const ModelParams& M, uint32_t it) {
  const uint32_t shift = M.D == 128 ? 3 : 2, row = it >> shift, tok = row / (uint32_t)M.Hkv;
  return {(int)tok, (int)(row - tok * M.Hkv), (int)(it & ((1u << shift) - 1))};
}

__global__ void __launch_bounds__(kThreads) packed_append_kernel(const PackedCacheParams p) {
  const ModelParams& M = p.m;
  const int bpr = M.D / 16;  // blocks per row: 4 or 8
  const uint32_t items = (uint32_t)p.total_q * M.Hkv * bpr;
  const __nv_bfloat16* in = blockIdx.y ? p.v_in : p.k_in;
  const float g = blockIdx.y ? p.v_scale : p.k_scale;
  for (uint32_t it = blockIdx.x * kThreads + threadIdx.x; it < items; it += gridDim.x * kThreads) {
    const Item at_item = item_of(M, it);
    const int blk = at_item.blk;
    const uint4* src = reinterpret_cast<const uint4*>(in) + (int64_t)it * 2;
    const uint4 u0 = src[0], u1 = src[1];
    const RowAt at = find_row(p, at_item.tok, at_item.kh);
    if (!at.ok) continue;
    const uint32_t w[8] = {u0.x, u0.y, u0.z, u0.w, u1.x, u1.y, u1.z, u1.w};
    float x[16];
    float a = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 f = unpack_bf16x2(w[k]);
      x[2 * k] = f.x;
      x[2 * k + 1] = f.y;
      a = fmaxf(a, fmaxf(fabsf(f.x), fabsf(f.y)));  // (NaN are no magnitudes; infinities take the largest codes)
    }
    uint16_t code;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(code) : "f"(0.f), "f"(__fdiv_rn(__fdiv_rn(a, g), 6.f)));
    const float s = __half2float(__ushort_as_half((unsigned short)(e4m3_to_half2(code) & 0xffff))) * g;
    const float inv = __fdiv_rn(1.f, s);
    uint32_t held[2] = {0, 0};
    if (s > 0.f) {  // (a scale of 0 holds zeros)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        float y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float y0 = x[2 * k + e] * inv;
          // (from 8 on the level is 6 whatever the residual)
          y[e] = fabsf(y0) < 8.f ? fmaf(fmaf(-y0, s, x[2 * k + e]), inv, y0) : y0;
        }
        uint32_t b;
        asm("{\n\t.reg .b8 t;\n\tcvt.rn.satfinite.e2m1x2.f32 t, %1, %2;\n\tcvt.u32.u8 %0, t;\n\t}" : "=r"(b) : "f"(y[1]), "f"(y[0]));
        held[k >> 2] |= b << (8 * (k & 3));
      }
    }
    uint8_t* slab = p.pool + at.slab + (blockIdx.y ? (int64_t)M.Hkv * M.P * (M.D / 2 + M.D / 16) : 0);
    *reinterpret_cast<uint2*>(slab + at.slot * (M.D / 2) + blk * 8) = make_uint2(held[0], held[1]);
    slab[M.P * (M.D / 2) + at.slot * bpr + blk] = (uint8_t)code;
  }
}

__global__ void __launch_bounds__(kThreads) packed_read_kernel(const PackedCacheParams p) {
  const ModelParams& M = p.m;
  const int bpr = M.D / 16;
  const uint32_t items = (uint32_t)p.total_q * M.Hkv * bpr;
  __nv_bfloat16* out = blockIdx.y ? p.v_out : p.k_out;
  const float g = blockIdx.y ? p.v_scale : p.k_scale;
  for (uint32_t it = blockIdx.x * kThreads + threadIdx.x; it < items; it += gridDim.x * kThreads) {
    const Item at_item = item_of(M, it);
    const int blk = at_item.blk;
    const RowAt at = find_row(p, at_item.tok, at_item.kh);
    if (!at.ok) continue;
    const uint8_t* slab = p.pool + at.slab + (blockIdx.y ? (int64_t)M.Hkv * M.P * (M.D / 2 + M.D / 16) : 0);
    const uint2 held = *reinterpret_cast<const uint2*>(slab + at.slot * (M.D / 2) + blk * 8);
    const uint32_t f = e4m3_to_half2(slab[M.P * (M.D / 2) + at.slot * bpr + blk]);
    const uint32_t f2 = low_twice(f);
    uint32_t o[8];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const uint32_t word = k ? held.y : held.x;
      const uint32_t h[4] = {hmul2(e2m1_to_half2<0>(word), f2), hmul2(e2m1_to_half2<1>(word), f2), hmul2(e2m1_to_half2<2>(word), f2),
                             hmul2(e2m1_to_half2<3>(word), f2)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        o[4 * k + i] = pack_bf16x2(v.x * g, v.y * g);
      }
    }
    uint4* dst = reinterpret_cast<uint4*>(out) + (int64_t)it * 2;
    dst[0] = make_uint4(o[0], o[1], o[2], o[3]);
    dst[1] = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

dim3 grid_of(const PackedCacheParams& p, int num_sms) {
  const int64_t items = (int64_t)p.total_q * p.m.Hkv * (p.m.D / 16), blocks = (items + kThreads - 1) / kThreads, most = 16LL * num_sms;
  return dim3((unsigned)(blocks < most ? blocks : most), 2, 1);
}

}  // namespace

cudaError_t hswa_launch_packed_append(const PackedCacheParams& p, int num_sms, cudaStream_t s) {
  packed_append_kernel<<<grid_of(p, num_sms), kThreads, 0, s>>>(p);
  return cudaGetLastError();
}
cudaError_t hswa_launch_packed_read(const PackedCacheParams& p, int num_sms, cudaStream_t s) {
  packed_read_kernel<<<grid_of(p, num_sms), kThreads, 0, s>>>(p);
  return cudaGetLastError();
}
