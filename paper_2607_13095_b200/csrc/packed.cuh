// A Full layer's cache in 4 bits: the pool's layout, kernel parameters and the conversions that its kernels share.
//
// A row of D elements is held as D / 2 bytes (e2m1, the even element in the low half) and D / 16 e4m3 scales; a slab, one
// (page, K|V, head), is the P rows' bytes and then the P rows' scales.  e2m1 has at most 2 significant bits and e4m3 at most
// 4, with products between 2^-10 and 2688: a held value e2m1 * e4m3 is exact in fp16 (and bf16), so the tensor cores multiply
// the held values themselves; the layer's two fp32 scales are applied to scores and outputs.
#pragma once

#include <cuda_fp16.h>

#include "hswa_internal.cuh"

struct PackedCacheParams {  // append and read-back
  ModelParams m;
  BatchParams b;
  uint8_t* pool;  // [num_pages][2][Hkv][P * (D / 2 + D / 16)]
  int64_t num_pages;
  float k_scale, v_scale;
  const __nv_bfloat16* k_in;  // [T][Hkv][D] (append)
  const __nv_bfloat16* v_in;
  __nv_bfloat16* k_out;  // [T][Hkv][D] (read-back)
  __nv_bfloat16* v_out;
  int32_t total_q, max_q_len, max_ctx_len;
  int32_t* err;
};

struct PackedAttnParams {
  ModelParams m;
  BatchParams b;
  const uint8_t* pool;
  int64_t num_pages;
  float scale_log2;  // sm_scale * log2(e) * k_scale
  float v_scale;
  int32_t causal;
  const __nv_bfloat16* q;  // [T][Hq][D]
  void* out;               // [T][Hq][D]
  float* lse;              // [T][Hq] or null
  int32_t total_q, max_q_len, max_ctx_len;
  // few rows: runs of tiles (0: a block per stream) and the tiles of all requests before each, [B + 1]
  int32_t runs;
  int64_t* before;
  // many rows: blocks along a request's rows, keys per slice (a multiple of 128), slices per row
  int32_t row_tiles, slice_len, slices;
  float* part_o;    // few rows: [2 runs][rows of a block][D]; many: [T * Hq][slices][D]
  float2* part_ml;  // the same without D: (m in log2 units, l)
  int32_t* err;
};

cudaError_t hswa_launch_packed_append(const PackedCacheParams& p, int num_sms, cudaStream_t s);
cudaError_t hswa_launch_packed_read(const PackedCacheParams& p, int num_sms, cudaStream_t s);
// Up to eight rows (tokens x heads of a KV head), long contexts: a run per warp
int hswa_packed_stream_runs_per_sm();
cudaError_t hswa_launch_packed_stream(const PackedAttnParams& p, cudaStream_t s);
// Few rows, long contexts, on the 5th-generation tensor cores: up to 16 or 32 rows, a run per SM
// (tm_pool: the pool as {slab / 9, 9, Hkv, 2, pages}, box of a page's K and V of one head)
cudaError_t hswa_launch_packed_rows(const CUtensorMap& tm_pool, const PackedAttnParams& p, int rows, cudaStream_t s);
// The join of runs' pieces of `cols` rows each over key tiles of `tile`
cudaError_t hswa_launch_packed_join(const PackedAttnParams& p, int cols, int tile, cudaStream_t s);
// Up to 8, 16 or 32 rows, short contexts: a block per stream
cudaError_t hswa_launch_packed_decode(const PackedAttnParams& p, int rows, cudaStream_t s);
// Many rows: the tcgen05 tile kernel, two Q tiles of hswa_cross_tile_tokens tokens per block
cudaError_t hswa_launch_packed_tile(const PackedAttnParams& p, cudaStream_t s);

#ifdef __CUDACC__
namespace hswa_dev {

// Two e2m1 values (one byte) to fp16; the low half of the byte goes to the low half of the result.
template <int BYTE>
__device__ __forceinline__ uint32_t e2m1_to_half2(uint32_t w) {
  uint32_t r;
  if constexpr (BYTE == 0)
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(r) : "r"(w));
  else if constexpr (BYTE == 1)
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(r) : "r"(w));
  else if constexpr (BYTE == 2)
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(r) : "r"(w));
  else
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, d;\n\t}" : "=r"(r) : "r"(w));
  return r;
}
// Two e4m3 values (the low 16 bits) to fp16.
__device__ __forceinline__ uint32_t e4m3_to_half2(uint32_t w) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
  return r;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t low_twice(uint32_t a) { return __byte_perm(a, a, 0x1010); }
__device__ __forceinline__ uint32_t high_twice(uint32_t a) { return __byte_perm(a, a, 0x3232); }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// D(16x8, fp32) += A(16x16, fp16, row) * B(16x8, fp16, col)
__device__ __forceinline__ void mma_f16_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                              uint32_t b1) {
  asm(  // (not volatile: independent products may be interleaved)
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same from zero
__device__ __forceinline__ void mma_f16_16816_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                                   uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

// Probabilities enter the PV product as fp16, whose 11 bits are rounding enough for outputs in bf16, but whose exponents end at 2^-24: they
// are taken relative to a base 2^7 below the row's maximum, and the base moves when a score passes it by more than 2^15, the most that
// fp16 holds.  What a key adds is then off by 2^-11 of itself or, below 2^-21 of the row's largest, by 2^-32 of that.  (Relative to the
// maximum itself, 2^-25: a million keys 25 bits below one of them would lose 3 % of the row's weight.)  The base of a tile's largest score `top`
// (times `mul`, in log2 units), and whether a row moves to it; the 2^-22 covers the roundings of large scores.
constexpr float kBaseBelowMax = 7.f, kMostAboveBase = 15.f;
__device__ __forceinline__ float base_of(float top, float mul) { return fmaf(top, mul, -kBaseBelowMax); }
__device__ __forceinline__ bool base_moves(float to, float from) {
  return fmaf(fabsf(to), 0x1p-22f, to) > from + (kMostAboveBase - kBaseBelowMax);  // (never to minus infinity)
}

// Queries enter the products as fp16, each row times a power of two that brings its largest element to [2^14, 2^15): fp16
// has three bits more than bf16, so only elements below 2^-28 of the largest lose any.  (Rows below 2^-112 are multiplied by 2^126, the
// largest whose inverse is a normal number: their elements, down to bf16's smallest, stay normal in fp16.)  From the largest magnitude,
// infinities and NaN apart, the power and its inverse.
__device__ __forceinline__ float finite_max(float amax, float2 f) {
  const float a = fabsf(f.x), b = fabsf(f.y);
  return fmaxf(amax, fmaxf(a < INFINITY ? a : 0.f, b < INFINITY ? b : 0.f));
}
__device__ __forceinline__ void q_powers(float amax, float* up, float* down) {
  const int e = (int)(__float_as_uint(amax) >> 23);  // biased exponent
  const int shift = amax > 0.f ? min(141 - e, 126) : 0;
  *up = __uint_as_float((uint32_t)(127 + shift) << 23);
  *down = __uint_as_float((uint32_t)(127 - shift) << 23);
}

__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap* tm, uint32_t bar, int c0, int c1, int c2, int c3, int c4) {
  asm volatile(
      "cp.async.bulk.tensor.5d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst), "l"(tm),
      "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4)
      : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
               "r"(bytes), "r"(bar)
               : "memory");
}

}  // namespace hswa_dev
#endif  // __CUDACC__
