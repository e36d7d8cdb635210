// Rows into and out of a 4-bit cache (hswa_packed_append, hswa_packed_read): two neighbouring lanes per block of 16 elements, so that
// a warp's 16-byte loads and stores follow one another.
//
// A block of 16 elements x with largest magnitude a, in a layer of scale g, is held as f = e4m3((a / g) / 6), s = f g, and
// e2m1(x / s): both roundings to the nearest, ties to the even code, at most 448 and 6.  Quotients lie halfway between two codes
// often (dividend and divisor have few bits), so they have to be right to the last bit: a product with the inverse, then one
// Newton step on its exact residual, which makes every quotient exact that fits 24 bits.  (Layer scales of more than 14 bits make other
// quotients, which 32 bits may round to a half: within 2^-22 of one either code may be held.)  (Divisions take the append from 59
// to 79 us; a pair of elements per instruction, from 52 to 46.)
// Bound by HBM (2 bytes per element read, 0.5625 written; read-back: the reverse) and by issue: 70 % of the slots at ten
// instructions an element.  A block takes some tokens: it looks up where their rows are held (a chain of dependent loads) once, and then
// moves their elements with several loads in flight; a thread that looked up its own row was at half the rate.  Measured, 8 prompts of
// up to 8192 tokens, 8 KV heads of 128 (200 MB each way, floor 30 us): append 46 us, read-back 35; with 32 tokens a block 47 and 36 (fewer,
// longer blocks end less evenly).
#include "packed.cuh"

namespace {
using namespace hswa_dev;

constexpr int kThreads = 256;
constexpr int kTokens = 16;  // of a block, at most
constexpr int kAtOnce = 4;   // items that a thread has in flight

struct RowAt {
  uint8_t *values, *scales;  // of KV head 0, K or V as the block moves; null: not to be moved
};

// Where the row of token `tok` (of all requests' tokens) is held; records what is out of range.
__device__ __forceinline__ RowAt find_row(const PackedCacheParams& p, int tok) {
  const ModelParams& M = p.m;
  RowAt at = {nullptr, nullptr};
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
  const int slot = pos - block * M.P;
  uint8_t* slab = p.pool + ((int64_t)page * 2 + blockIdx.y) * M.Hkv * (M.P * (M.D / 2 + M.D / 16));
  at.values = slab + slot * (M.D / 2);
  at.scales = slab + M.P * (M.D / 2) + slot * (M.D / 16);
  return at;
}

// The rows of the block's tokens [tok0, tok0 + n).
__device__ __forceinline__ int find_rows(const PackedCacheParams& p, int tokens, RowAt* s_at) {
  const int tok0 = blockIdx.x * tokens, n = min(tokens, p.total_q - tok0);
  if (threadIdx.x < n) s_at[threadIdx.x] = find_row(p, tok0 + threadIdx.x);
  __syncthreads();
  return n;
}

// What a thread's items have in common: item `it` of the block is eight elements, half of a block of 16, of row it / (D / 8) of the
// block's tokens and KV heads; a thread's items are kThreads, a multiple of D / 8, apart, so all are the same part of their rows.
struct Part {
  int shift;
  uint32_t values, scale, slab;  // byte offsets in a row and its scales, bytes of a slab
};
__device__ __forceinline__ Part part_of(const PackedCacheParams& p) {
  const ModelParams& M = p.m;
  const int shift = M.D == 128 ? 4 : 3;
  const uint32_t oct = threadIdx.x & ((1u << shift) - 1);
  return {shift, oct * 4, oct / 2, (uint32_t)(M.P * (M.D / 2 + M.D / 16))};
}
__device__ __forceinline__ RowAt item_of(const PackedCacheParams& p, const RowAt* s_at, const Part& part, uint32_t it, uint32_t per_head) {
  const uint32_t heads = p.m.Hkv, row = it >> part.shift, tok = heads == 1 ? row : __umulhi(row, per_head), kh = row - tok * heads;
  RowAt at = s_at[tok];
  if (at.values) {
    at.values += kh * part.slab + part.values;
    at.scales += kh * part.slab + part.scale;
  }
  return at;
}

// x / d from inv = 1 / d to a few last places; infinite products stay what they are.
__device__ __forceinline__ float quotient(float x, float d, float inv) {
  const float q = x * inv;
  return fabsf(q) < 3e38f ? fmaf(fmaf(-q, d, x), inv, q) : q;
}
__device__ __forceinline__ float2 quotient_below_max(float2 x, float2 minus_d, float2 inv) {  // (of finite products)
  const float2 q = __fmul2_rn(x, inv);
  return __ffma2_rn(__ffma2_rn(q, minus_d, x), inv, q);
}
// Eight elements to codes; the lane beside has the other half of the block.
__device__ __forceinline__ uint32_t to_codes(const uint4 u, float g, float inv_g, uint16_t* code_out) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
  float2 x[4];
  float a = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[k] = unpack_bf16x2(w[k]);
    a = fmaxf(a, fmaxf(fabsf(x[k].x), fabsf(x[k].y)));  // (NaN are no magnitudes; infinities take the largest codes)
  }
  a = fmaxf(a, __shfl_xor_sync(0xffffffffu, a, 1));
  uint16_t code;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(code) : "f"(0.f), "f"(quotient(quotient(a, g, inv_g), 6.f, 1.f / 6.f)));
  *code_out = code;
  const float s = __half2float(__ushort_as_half((unsigned short)(e4m3_to_half2(code) & 0xffff))) * g;
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
  float2 y[4];
  if (code == 0x7e) {  // 448: elements may lie far above 6 s
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = make_float2(quotient(x[k].x, s, inv), quotient(x[k].y, s, inv));
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) y[k] = quotient_below_max(x[k], make_float2(-s, -s), make_float2(inv, inv));
  }
  uint32_t held;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(held)
      : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
  return s > 0.f ? held : 0;  // (a scale of 0 holds zeros)
}

__global__ void __launch_bounds__(kThreads) packed_append_kernel(const PackedCacheParams p, const int tokens, const uint32_t per_head) {
  __shared__ RowAt s_at[kTokens];
  const ModelParams& M = p.m;
  const int n = find_rows(p, tokens, s_at);
  const uint32_t items = (uint32_t)n * M.Hkv * (M.D / 8);
  const Part part = part_of(p);
  const uint4* in = reinterpret_cast<const uint4*>((blockIdx.y ? p.v_in : p.k_in) + (int64_t)blockIdx.x * tokens * M.Hkv * M.D);
  const float g = blockIdx.y ? p.v_scale : p.k_scale, inv_g = __fdiv_rn(1.f, g);
  for (uint32_t base = 0; base < items; base += kAtOnce * kThreads) {
    uint4 u[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t it = base + k * kThreads + threadIdx.x;
      u[k] = it < items ? in[it] : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (base + k * kThreads >= items) break;  // (uniform)
      const uint32_t it = base + k * kThreads + threadIdx.x;
      uint16_t code;
      const uint32_t held = to_codes(u[k], g, inv_g, &code);
      if (it >= items) continue;
      const RowAt at = item_of(p, s_at, part, it, per_head);
      if (!at.values) continue;
      *reinterpret_cast<uint32_t*>(at.values) = held;
      if (!(it & 1)) *at.scales = (uint8_t)code;
    }
  }
}

__global__ void __launch_bounds__(kThreads) packed_read_kernel(const PackedCacheParams p, const int tokens, const uint32_t per_head) {
  __shared__ RowAt s_at[kTokens];
  const ModelParams& M = p.m;
  const int n = find_rows(p, tokens, s_at);
  const uint32_t items = (uint32_t)n * M.Hkv * (M.D / 8);
  const Part part = part_of(p);
  uint4* out = reinterpret_cast<uint4*>((blockIdx.y ? p.v_out : p.k_out) + (int64_t)blockIdx.x * tokens * M.Hkv * M.D);
  const float g = blockIdx.y ? p.v_scale : p.k_scale;
  for (uint32_t it0 = threadIdx.x; it0 < items; it0 += kAtOnce * kThreads) {
    uint32_t held[kAtOnce], code[kAtOnce];
    bool there[kAtOnce];
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      const uint32_t it = it0 + k * kThreads;
      there[k] = false;
      if (it >= items) continue;
      const RowAt at = item_of(p, s_at, part, it, per_head);
      there[k] = at.values != nullptr;
      if (!there[k]) continue;
      held[k] = *reinterpret_cast<const uint32_t*>(at.values);
      code[k] = *at.scales;
    }
#pragma unroll
    for (int k = 0; k < kAtOnce; ++k) {
      if (!there[k]) continue;
      const uint32_t f2 = low_twice(e4m3_to_half2(code[k])), w = held[k];
      const uint32_t h[4] = {hmul2(e2m1_to_half2<0>(w), f2), hmul2(e2m1_to_half2<1>(w), f2), hmul2(e2m1_to_half2<2>(w), f2),
                             hmul2(e2m1_to_half2<3>(w), f2)};
      uint32_t o[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = __fmul2_rn(__half22float2(*reinterpret_cast<const __half2*>(&h[i])), make_float2(g, g));
        o[i] = pack_bf16x2(v.x, v.y);
      }
      out[it0 + k * kThreads] = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// Tokens of a block: enough for a few rounds of its threads, and blocks enough for the SMs.
struct Geometry {
  int tokens;
  dim3 grid;
  uint32_t per_head;  // 2^32 / Hkv, rounded up: a row's token by one multiplication (exact while row and Hkv are below 2^16)
};
Geometry geometry(const PackedCacheParams& p, int num_sms) {
  const int per_token = p.m.Hkv * (p.m.D / 8);
  int tokens = 2 * kAtOnce * kThreads / per_token;
  const int most = p.total_q / (2 * num_sms);
  tokens = tokens > most ? most : tokens;
  tokens = tokens < 1 ? 1 : tokens > kTokens ? kTokens : tokens;
  return {tokens, dim3((unsigned)((p.total_q + tokens - 1) / tokens), 2, 1), p.m.Hkv == 1 ? 0 : (uint32_t)((1ull << 32) / p.m.Hkv + 1)};
}

}  // namespace

cudaError_t hswa_launch_packed_append(const PackedCacheParams& p, int num_sms, cudaStream_t s) {
  const Geometry g = geometry(p, num_sms);
  packed_append_kernel<<<g.grid, kThreads, 0, s>>>(p, g.tokens, g.per_head);
  return cudaGetLastError();
}
cudaError_t hswa_launch_packed_read(const PackedCacheParams& p, int num_sms, cudaStream_t s) {
  const Geometry g = geometry(p, num_sms);
  packed_read_kernel<<<g.grid, kThreads, 0, s>>>(p, g.tokens, g.per_head);
  return cudaGetLastError();
}
