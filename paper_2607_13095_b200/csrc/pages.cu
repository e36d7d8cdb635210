// Bookkeeping of a cache's pages on the device: hswa_pages_fork, hswa_pages_compact, hswa_pages_copy.
//
// Counts (how many holders a page has) are the only state: a page of count 0 is free, and the lowest-numbered free pages are
// taken first, so results depend on the counts alone.  The steps that depend on one another (ranks of free and live pages, what each
// row needs) are one launch of one cluster of 16 blocks, whose barrier between two steps costs a fraction of a launch: each block
// turns its share of the counts into a bitmap in shared memory on the only pass over them, ranks come from the bitmap, and totals
// go around through distributed shared memory.  Of a large pool all SMs make the bitmap, by a launch before the cluster's, which overlaps
// with its look at the rows (512 rows, a million counts: 20 us a fork, 24 where the cluster reads the counts itself).  Rewriting the
// tables is the cluster's work as well while they are small; large ones are rewritten by a second launch of all SMs (a million
// entries: 66 us by 16 SMs, 22 with the second launch).  Bound by latency: launches, barriers and a chain of dependent loads; 8 rows
// over 2048 pages take 9.4 us (fork) and 7.5 (compact).
#include <cooperative_groups.h>

#include <utility>

#include "pages.cuh"

namespace {
using namespace hswa_dev;
namespace cg = cooperative_groups;

constexpr int kBlocks = 16;     // blocks of the cluster
constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;

// A block's share of the pages: words [first, first + words) of 32 pages each.
struct Share {
  int first, words;
};
__device__ __forceinline__ Share share_of(int num_pages, int block) {
  const int all = (num_pages + 31) / 32, per = (all + kBlocks - 1) / kBlocks;
  Share s;
  s.first = min(block * per, all);
  s.words = min(per, all - s.first);
  return s;
}

// Exclusive prefix sum of `mine` over the block's threads; `total` gets the sum of all.
__device__ __forceinline__ int block_prefix(int mine, int* s_warp, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = mine;
#pragma unroll
  for (int sh = 1; sh < 32; sh <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, incl, sh);
    if (lane >= sh) incl += v;
  }
  __syncthreads();  // (s_warp of an earlier call has been read)
  if (lane == 31) s_warp[warp] = incl;
  __syncthreads();
  int w = lane < kWarps ? s_warp[lane] : 0, wi = w;
#pragma unroll
  for (int sh = 1; sh < 32; sh <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, wi, sh);
    if (lane >= sh) wi += v;
  }
  *total = __shfl_sync(0xffffffffu, wi, 31);
  return __shfl_sync(0xffffffffu, wi - w, warp) + incl - mine;
}

// The block's share of the counts on its way to L2, while the rows are looked at.
__device__ __forceinline__ void fetch_counts(const int32_t* ref, int num_pages, Share sh) {
  for (int w = threadIdx.x; w < sh.words; w += kThreads)
    if ((sh.first + w) * 32 < num_pages) asm volatile("prefetch.global.L2 [%0];" ::"l"(ref + (int64_t)(sh.first + w) * 32));
}
// The one pass over the counts, by warp `warp` of `warps`: sets the bit of every free page and copies the counts; `map`, where given, gets
// the identity from entry `map_from` on.  U: loads in flight, 16 bytes, four pages, of each lane; a warp's load covers four words of the
// bitmap.
template <int U>
__device__ __forceinline__ void scan_counts(const int32_t* ref, int32_t* ref_out, int32_t* map, int map_from, int num_pages, Share sh,
                                            uint32_t* free_bits, int warp, int warps) {
  const int lane = threadIdx.x & 31;
  const bool wide = ((reinterpret_cast<uintptr_t>(ref) | reinterpret_cast<uintptr_t>(ref_out) | reinterpret_cast<uintptr_t>(map)) & 15) == 0;
  for (int w0 = warp * 4 * U; w0 < sh.words; w0 += warps * 4 * U) {
    int4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t page = (int64_t)(sh.first + w0 + 4 * u) * 32 + 4 * lane;
      if (w0 + 4 * u + lane / 8 >= sh.words) {
        v[u] = make_int4(1, 1, 1, 1);  // (another block's)
      } else if (wide && page + 4 <= num_pages) {
        v[u] = *reinterpret_cast<const int4*>(ref + page);
      } else {
        v[u].x = page < num_pages ? ref[page] : 1;  // (no page: not a free one)
        v[u].y = page + 1 < num_pages ? ref[page + 1] : 1;
        v[u].z = page + 2 < num_pages ? ref[page + 2] : 1;
        v[u].w = page + 3 < num_pages ? ref[page + 3] : 1;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int word = w0 + 4 * u + lane / 8;
      const int64_t page = (int64_t)(sh.first + w0 + 4 * u) * 32 + 4 * lane;
      uint32_t bits = (uint32_t)(v[u].x <= 0) | (uint32_t)(v[u].y <= 0) << 1 | (uint32_t)(v[u].z <= 0) << 2 | (uint32_t)(v[u].w <= 0) << 3;
      bits <<= 4 * (lane & 7);
#pragma unroll
      for (int x = 1; x < 8; x <<= 1) bits |= __shfl_xor_sync(0xffffffffu, bits, x);
      if (word >= sh.words) continue;
      if ((lane & 7) == 0) free_bits[word] = bits;
      if (wide && page + 4 <= num_pages && (!map || page >= map_from)) {
        *reinterpret_cast<int4*>(ref_out + page) = v[u];
        if (map) *reinterpret_cast<int4*>(map + page) = make_int4((int)page, (int)page + 1, (int)page + 2, (int)page + 3);
      } else {
        const int32_t each[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (page + e >= num_pages) break;
          ref_out[page + e] = each[e];
          if (map && page + e >= map_from) map[page + e] = (int)page + e;
        }
      }
    }
  }
}
// The pages of a word that are there.
__device__ __forceinline__ uint32_t pages_of_word(int num_pages, int word) {
  const int left = num_pages - word * 32;
  return left >= 32 ? 0xffffffffu : (1u << left) - 1;
}

// Sums a per-block number over the blocks before this one and over all of them.  `started`: what the block's arrival at the
// kernel's start gave (a block's shared memory may be written by another once it runs).
__device__ __forceinline__ void cluster_prefix(cg::cluster_group& cluster, cg::cluster_group::arrival_token&& started, int mine,
                                               int* s_counts, int* before, int* all) {
  cluster.barrier_wait(std::move(started));
  if (threadIdx.x < kBlocks) *cluster.map_shared_rank(&s_counts[cluster.block_rank()], threadIdx.x) = mine;
  cluster.sync();
  int b = 0, a = 0;
  for (int i = 0; i < kBlocks; ++i) {
    a += s_counts[i];
    if (i < (int)cluster.block_rank()) b += s_counts[i];
  }
  *before = b;
  *all = a;
}

// The pass over the counts of a large pool by all SMs, while the cluster behind it looks at the rows.  Where given, `map` gets the identity,
// but for its first entries if the bitmap lies there: the cluster, which reads the bitmap, sets those.
constexpr int kWideThreads = 256;
__global__ void __launch_bounds__(kWideThreads) pages_copy_counts_kernel(const int32_t* ref, int32_t* ref_out, int32_t* map, uint32_t* bits,
                                                                         const int num_pages) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const Share all = {0, (num_pages + 31) / 32};
  scan_counts<2>(ref, ref_out, map, all.words, num_pages, all, bits, blockIdx.x * (kWideThreads / 32) + (threadIdx.x >> 5),
                 gridDim.x * (kWideThreads / 32));
}
// The block's part of that bitmap; `map`: the first entries, where it lies, get the identity.
__device__ __forceinline__ void take_bits(const uint32_t* bits, int32_t* map, Share sh, uint32_t* free_bits) {
  for (int w = threadIdx.x; w < sh.words; w += kThreads) {
    free_bits[w] = bits[sh.first + w];
    if (map) map[sh.first + w] = sh.first + w;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Fork.  Row r of the new tables continues row parent[r] of the old ones at len[r] tokens.  Its first len / P pages are shared;
// of the places from there on, the ones whose page the parent alone holds and no child shares go on with the parent's first
// child, and all others get fresh pages.  What the rules need of the old counts is decided before the barrier and kept as the
// rank of a row's first fresh page; the counts of pages change behind it, by atomic adds whose order does not matter.
// ---------------------------------------------------------------------------------------------------------------------
struct RowPlan {
  int parent, full, held, parent_held, most;  // shared pages, pages of the row, pages of its parent, most pages that a child of it shares
  bool first;                                 // the parent's first child
};
__device__ __forceinline__ int pages_of(int tokens, int page_size) { return (int)(((int64_t)tokens + page_size - 1) / page_size); }
// The rows' arrays: the call's own, or their copies in shared memory.
struct Rows {
  const int32_t *parent, *len, *need, *held, *first, *most, *rank;
};
__device__ __forceinline__ RowPlan plan_of(const PagesForkParams& p, const Rows& rows, int r) {
  RowPlan o;
  o.parent = rows.parent[r];
  const int len = rows.len[r];
  o.full = len / p.page_size;
  o.held = pages_of(max(len, rows.need[r]), p.page_size);
  o.parent_held = o.parent >= 0 ? rows.held[o.parent] : 0;
  o.first = o.parent >= 0 && rows.first[o.parent] == r;
  o.most = o.parent >= 0 ? rows.most[o.parent] : 0;
  return o;
}
// Does place k >= full of the row keep the parent's page?
__device__ __forceinline__ bool passed(const PagesForkParams& p, const RowPlan& o, int k, int* page_out) {
  if (!o.first || k >= o.parent_held || k < o.most) return false;
  const int page = p.table[(int64_t)o.parent * p.max_blocks + k];
  *page_out = page;
  return page >= 0 && page < p.num_pages && p.ref[page] == 1;
}

// The new tables and counts, by warp `me` of `all`: the rows' plans are made, fresh pages listed, counts copied.
__device__ __forceinline__ void apply_fork(const PagesForkParams& p, const Rows& rows, int me, int all) {
  const int lane = threadIdx.x & 31;
  auto count = [&](int page, int by, int row, int k) {
    if (page < 0 || page >= p.num_pages)
      record_error(p.err, HSWA_ERR_BOUNDS, row, k, page);
    else if (by != 0)
      atomicAdd(&p.ref_out[page], by);
  };
  constexpr int CH = 256;  // places per item
  const int chunks = max(1, (max(p.max_blocks, p.out_max_blocks) + CH - 1) / CH);  // (tables without places have rows all the same)
  // new rows: shared places in chunks of 256, the places behind them by the warp of chunk 0
  for (int64_t it = me; it < (int64_t)p.rows_out * chunks; it += all) {
    const int r = (int)(it / chunks), c = (int)(it % chunks);
    const RowPlan o = plan_of(p, rows, r);
    int32_t* out = p.table_out + (int64_t)r * p.out_max_blocks;
    const int32_t* in = p.table + (int64_t)max(o.parent, 0) * p.max_blocks;
    int page[CH / 32];
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      page[u] = k < o.full ? in[k] : 0;
    }
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      if (k >= o.full) continue;
      out[k] = page[u];
      count(page[u], o.first ? 0 : 1, r, k);
    }
    if (c != 0) continue;
    int next = rows.rank[r];
    const int len = rows.len[r];
    int src = -1, dst = -1;
    for (int k0 = o.full; k0 < o.held; k0 += 32) {
      const int k = k0 + lane;
      int at = -1;
      const bool keeps = k < o.held && passed(p, o, k, &at);
      const bool fresh = k < o.held && !keeps;
      const uint32_t who = __ballot_sync(0xffffffffu, fresh);
      if (fresh) {
        at = p.fresh[next + __popc(who & ((1u << lane) - 1))];
        p.ref_out[at] = 1;
      }
      if (k < o.held) out[k] = at;
      next += __popc(who);
      if (k == o.full && fresh && len % p.page_size != 0) {
        src = in[k];
        dst = at;
        if (src < 0 || src >= p.num_pages) {
          record_error(p.err, HSWA_ERR_BOUNDS, r, k, src);
          src = dst = -1;
        }
      }
    }
    if (lane == 0) {  // (place `full` is lane 0's)
      p.copy_src[r] = src;
      p.copy_dst[r] = dst;
      p.held_out[r] = o.held;
    }
  }
  // old rows: what their first child does not keep loses a holder
  for (int64_t it = me; it < (int64_t)p.rows_in * chunks; it += all) {
    const int i = (int)(it / chunks), c = (int)(it % chunks);
    const int held = rows.held[i], child = rows.first[i];
    RowPlan o = {};
    if (child != INT32_MAX) o = plan_of(p, rows, child);
    if (child != INT32_MAX && min(held, (c + 1) * CH) <= o.full) continue;
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      if (k >= held || (child != INT32_MAX && k < o.full)) continue;
      int page;
      if (child != INT32_MAX && k < o.held && passed(p, o, k, &page)) continue;
      count(p.table[(int64_t)i * p.max_blocks + k], -1, i, k);
    }
  }
}

__global__ void __launch_bounds__(kThreads) pages_fork_kernel(const PagesForkParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  auto started = cluster.barrier_arrive();
  extern __shared__ int32_t s_mem[];
  __shared__ int s_warp[kWarps], s_counts[kBlocks];
  int32_t* s_first = s_mem;                 // [rows_in] first child
  int32_t* s_most = s_first + p.rows_in;    // [rows_in] most pages that a child shares
  int32_t* s_held = s_most + p.rows_in;     // [rows_in]
  int32_t* s_rank = s_held + p.rows_in;     // [rows_out] rank of the row's first fresh page
  int32_t* s_parent = s_rank + p.rows_out;  // [rows_out] and two more
  int32_t* s_len = s_parent + p.rows_out;
  int32_t* s_need = s_len + p.rows_out;
  uint32_t* s_free = reinterpret_cast<uint32_t*>(s_need + p.rows_out);
  const Rows rows = {s_parent, s_len, s_need, s_held, s_first, s_most, s_rank};
  const int block = (int)cluster.block_rank(), warp = threadIdx.x >> 5;
  const Share sh = share_of(p.num_pages, block);
  if (p.second) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (else another handle's decode may follow, and read early)
  if (!p.copied) fetch_counts(p.ref, p.num_pages, sh);
  bool bad = false;
  for (int i = threadIdx.x; i < p.rows_in; i += kThreads) {
    const int held = p.held[i];
    s_first[i] = INT32_MAX;
    s_most[i] = 0;
    s_held[i] = held;
    if (held < 0 || held > p.max_blocks) {
      bad = true;
      if (block == 0) record_error(p.err, HSWA_ERR_BOUNDS, i, -1, held);
    }
  }
  for (int r = threadIdx.x; r < p.rows_out; r += kThreads) {
    s_parent[r] = p.parent[r];
    s_len[r] = p.len[r];
    s_need[r] = p.need[r];
  }
  // every block looks at all rows, so none waits for another, and all come to the same answer: the votes are barriers as well
  bad = __syncthreads_or(bad);
  for (int r = threadIdx.x; r < p.rows_out; r += kThreads) {
    const int parent = s_parent[r], len = s_len[r], need = s_need[r];
    bool ok = parent >= -1 && parent < p.rows_in && len >= 0 && pages_of(max(len, need), p.page_size) <= p.out_max_blocks;
    if (ok) ok = parent < 0 ? len == 0 : pages_of(len, p.page_size) <= s_held[parent];
    if (!ok) {
      bad = true;
      if (block == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, -2, parent);
    } else if (parent >= 0) {
      atomicMin(&s_first[parent], r);
      atomicMax(&s_most[parent], len / p.page_size);
    }
  }
  const bool rows_ok = !__syncthreads_or(bad);
  int fresh_total = 0;
  if (rows_ok) {
    const int per = (p.rows_out + kThreads - 1) / kThreads;
    const int r0 = threadIdx.x * per, r1 = min(r0 + per, p.rows_out);
    int sum = 0;
    for (int r = r0; r < r1; ++r) {
      const RowPlan o = plan_of(p, rows, r);
      int fresh = o.held - o.full, page;
      for (int k = o.most; o.first && k < min(o.held, o.parent_held); ++k) fresh -= passed(p, o, k, &page);
      s_rank[r] = sum;
      sum += fresh;
    }
    const int before = block_prefix(sum, s_warp, &fresh_total);
    for (int r = r0; r < r1; ++r) s_rank[r] += before;
  }

  // the free pages of lowest number
  asm volatile("griddepcontrol.wait;" ::: "memory");  // (with p.copied: the pass over the counts, launched before, is done)
  if (p.copied) take_bits(reinterpret_cast<const uint32_t*>(p.fresh), nullptr, sh, s_free);
  else scan_counts<4>(p.ref, p.ref_out, nullptr, 0, p.num_pages, sh, s_free, warp, kWarps);
  __syncthreads();
  const int wper = (sh.words + kThreads - 1) / kThreads;
  const int w0 = threadIdx.x * wper, w1 = min(w0 + wper, sh.words);
  int free_mine = 0;
  for (int w = w0; w < w1; ++w) free_mine += __popc(s_free[w]);
  int free_block, base, free_all;
  int rank = block_prefix(free_mine, s_warp, &free_block);
  cluster_prefix(cluster, std::move(started), free_block, s_counts, &base, &free_all);
  const bool enough = fresh_total <= free_all;
  if (!enough && rows_ok && block == 0 && threadIdx.x == 0) record_error(p.err, HSWA_ERR_BOUNDS, -1, fresh_total, free_all);
  if (rows_ok && enough) {
    rank += base;
    for (int w = w0; w < w1 && rank < fresh_total; ++w) {
      uint32_t bits = s_free[w];
      for (; bits && rank < fresh_total; bits &= bits - 1) p.fresh[rank++] = (sh.first + w) * 32 + __ffs(bits) - 1;
    }
  }
  if (p.second) {  // a second launch does the rest
    if (block == 0) {
      for (int i = threadIdx.x; i < p.rows_in; i += kThreads) {
        p.first[i] = s_first[i];
        p.most[i] = s_most[i];
      }
      for (int r = threadIdx.x; r < p.rows_out; r += kThreads) p.rank[r] = s_rank[r];
      if (threadIdx.x == 0) *p.ok = rows_ok && enough;
    }
    cluster.sync();  // (nobody reads another block's shared memory any more)
    return;
  }
  cluster.sync();  // counts copied, fresh pages listed, and nobody reads another block's shared memory any more
  if (rows_ok && enough) apply_fork(p, rows, block + kBlocks * warp, kBlocks * kWarps);
}

__global__ void __launch_bounds__(kWideThreads) pages_fork_apply_kernel(const PagesForkParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched early behind pages_fork_kernel
  if (*p.ok == 0) return;
  const Rows rows = {p.parent, p.len, p.need, p.held, p.first, p.most, p.rank};
  apply_fork(p, rows, blockIdx.x + gridDim.x * (threadIdx.x >> 5), gridDim.x * (kWideThreads / 32));
}

// ---------------------------------------------------------------------------------------------------------------------
// Compact.  With L live pages, the i-th lowest free page below L takes the i-th highest live page (those lie at or past L).
// A page's rank follows from the number of live pages before it.
// ---------------------------------------------------------------------------------------------------------------------
// The tables under the new numbers, by warp `me` of `all`.
__device__ __forceinline__ void apply_compact(const PagesCompactParams& p, int me, int all) {
  const int lane = threadIdx.x & 31;
  constexpr int CH = 256;
  const int chunks = (p.max_blocks + CH - 1) / CH;
  for (int64_t it = me; it < (int64_t)p.rows * chunks; it += all) {
    const int r = (int)(it / chunks), c = (int)(it % chunks);
    const int held = p.held[r];
    if (held < 0 || held > p.max_blocks) {
      if (c == 0 && lane == 0) record_error(p.err, HSWA_ERR_BOUNDS, r, -1, held);
      continue;
    }
    if (c * CH >= held) continue;
    int page[CH / 32];
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      page[u] = k < held ? p.table[(int64_t)r * p.max_blocks + k] : 0;
    }
    int to[CH / 32];
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      const bool ok = page[u] >= 0 && page[u] < p.num_pages;
      if (k < held && !ok) record_error(p.err, HSWA_ERR_BOUNDS, r, k, page[u]);
      to[u] = ok ? p.page_map[page[u]] : page[u];
    }
#pragma unroll
    for (int u = 0; u < CH / 32; ++u) {
      const int k = c * CH + u * 32 + lane;
      if (k < held) p.table_out[(int64_t)r * p.max_blocks + k] = to[u];
    }
  }
}
__global__ void __launch_bounds__(kWideThreads) pages_compact_apply_kernel(const PagesCompactParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");  // launched early behind pages_compact_kernel
  apply_compact(p, blockIdx.x + gridDim.x * (threadIdx.x >> 5), gridDim.x * (kWideThreads / 32));
}

__global__ void __launch_bounds__(kThreads) pages_compact_kernel(const PagesCompactParams p) {
  cg::cluster_group cluster = cg::this_cluster();
  auto started = cluster.barrier_arrive();
  extern __shared__ int32_t s_mem[];
  __shared__ int s_warp[kWarps], s_counts[kBlocks];
  const int block = (int)cluster.block_rank(), warp = threadIdx.x >> 5;
  const Share sh = share_of(p.num_pages, block);
  uint32_t* s_free = reinterpret_cast<uint32_t*>(s_mem);
  int32_t* s_before = s_mem + sh.words;  // live pages before each word's
  if (p.second) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (else another handle's decode may follow, and read early)
  if (!p.copied) fetch_counts(p.ref, p.num_pages, sh);
  for (int i = block * kThreads + threadIdx.x; i < p.max_moves; i += kBlocks * kThreads) p.move_src[i] = p.move_dst[i] = -1;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // (with p.copied: the pass over the counts, launched before, is done)
  if (p.copied) take_bits(reinterpret_cast<const uint32_t*>(p.page_map), p.page_map, sh, s_free);
  else scan_counts<4>(p.ref, p.ref_out, p.page_map, 0, p.num_pages, sh, s_free, warp, kWarps);
  __syncthreads();
  const int wper = (sh.words + kThreads - 1) / kThreads;
  const int w0 = threadIdx.x * wper, w1 = min(w0 + wper, sh.words);
  int mine = 0;
  for (int w = w0; w < w1; ++w) mine += __popc(pages_of_word(p.num_pages, sh.first + w) & ~s_free[w]);
  int in_block, base, total;
  int before = block_prefix(mine, s_warp, &in_block);
  cluster_prefix(cluster, std::move(started), in_block, s_counts, &base, &total);
  before += base;  // live pages before this thread's first
  for (int w = w0; w < w1; ++w) {
    s_before[w] = before;
    before += __popc(pages_of_word(p.num_pages, sh.first + w) & ~s_free[w]);
  }
  __syncthreads();
  // The pages to move lie close together, in the words of one or two blocks: neighbouring words go to different warps, and a warp takes
  // the pages of a word at once.  (A thread per word: 1 us more, 4096 moves.)
  const int lane = threadIdx.x & 31;
  for (int c = 0; c < sh.words; c += kThreads) {
    const int w = c + lane * 32 + ((warp + lane) & 31), page0 = (sh.first + w) * 32;
    uint32_t free = 0, live = 0;
    int at0 = 0;  // live pages before the word's
    bool any = false;
    if (w < sh.words) {
      free = s_free[w];
      live = pages_of_word(p.num_pages, sh.first + w) & ~free;
      at0 = s_before[w];
      any = (free && page0 < total && page0 - at0 < p.max_moves) ||
            (live && page0 + 31 >= total && total - (at0 + __popc(live)) < p.max_moves);
    }
    for (uint32_t who = __ballot_sync(0xffffffffu, any); who; who &= who - 1) {
      const int from = __ffs(who) - 1, page = __shfl_sync(0xffffffffu, page0, from) + lane;
      const uint32_t is_free = __shfl_sync(0xffffffffu, free, from) >> lane & 1, lives = __shfl_sync(0xffffffffu, live, from);
      const int rank = __shfl_sync(0xffffffffu, at0, from) + __popc(lives & ((1u << lane) - 1));  // live pages before the lane's
      if (is_free) {  // free pages below the number of live ones
        if (page < total && page - rank < p.max_moves) p.move_dst[page - rank] = page;
      } else if (lives >> lane & 1) {  // live pages from there on, counted from the highest
        if (page >= total && total - 1 - rank < p.max_moves) p.move_src[total - 1 - rank] = page;
      }
    }
  }
  cluster.sync();
  for (int i = block * kThreads + threadIdx.x; i < p.max_moves; i += kBlocks * kThreads) {
    const int src = p.move_src[i], dst = p.move_dst[i];
    if (src < 0) continue;
    p.page_map[src] = dst;
    p.ref_out[dst] = p.ref[src];
    p.ref_out[src] = 0;
  }
  if (p.second) return;  // a second launch rewrites the tables
  cluster.sync();
  apply_compact(p, block + kBlocks * warp, kBlocks * kWarps);
}

// ---------------------------------------------------------------------------------------------------------------------
// Copy.  A block moves 32 KB of one page of one pool; bound by HBM.
// ---------------------------------------------------------------------------------------------------------------------
constexpr int kCopyThreads = 256, kCopyLoads = 8, kCopyBytes = kCopyThreads * kCopyLoads * 16;

__global__ void __launch_bounds__(kCopyThreads) pages_copy_kernel(const PagesCopyParams p, const int chunks) {
  const int64_t pair = blockIdx.x / chunks;
  const int chunk = (int)(blockIdx.x % chunks);
  const int src = p.src[pair], dst = p.dst[pair];
  if (src < 0 && dst < 0) return;  // a place without a pair
  if (src < 0 || src >= p.num_pages || dst < 0 || dst >= p.num_pages) {
    if (threadIdx.x == 0 && chunk == 0) record_error(p.err, HSWA_ERR_BOUNDS, (int)pair, src, dst);
    return;
  }
  uint8_t* pool = static_cast<uint8_t*>(p.pools[blockIdx.y]);
  const int64_t from = (int64_t)chunk * kCopyBytes + threadIdx.x * 16;
  const uint4* s = reinterpret_cast<const uint4*>(pool + (int64_t)src * p.page_bytes + from);
  uint4* d = reinterpret_cast<uint4*>(pool + (int64_t)dst * p.page_bytes + from);
  uint4 v[kCopyLoads];
#pragma unroll
  for (int i = 0; i < kCopyLoads; ++i)
    if (from + (int64_t)i * kCopyThreads * 16 < p.page_bytes) v[i] = s[i * kCopyThreads];
#pragma unroll
  for (int i = 0; i < kCopyLoads; ++i)
    if (from + (int64_t)i * kCopyThreads * 16 < p.page_bytes) d[i * kCopyThreads] = v[i];
}

template <auto Kernel, typename Params>
cudaError_t launch_cluster(const Params& p, size_t smem, cudaStream_t s) {
  constexpr int most = kMaxPageRows * 7 * 4 + (kMaxPages / 32 / kBlocks) * 4;  // what the largest call needs
  static_assert(most <= 227 * 1024 - 1024, "rows and bitmap fit a block's shared memory");
  const cudaError_t e = hswa_prepare_kernel<Kernel>(most, true);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kBlocks, 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kBlocks;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = p.copied ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, Kernel, p);
}

// The second launch of all SMs, early behind the cluster.
template <typename Kernel, typename Params>
cudaError_t launch_wide(Kernel kern, const Params& p, int num_sms, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(4 * num_sms, 1, 1);
  cfg.blockDim = dim3(kWideThreads, 1, 1);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kern, p);
}

// Table entries up to which the cluster rewrites them itself, and pages up to which it copies the counts.
constexpr int64_t kSmallTables = 32768;
constexpr int kSmallPool = 65536;

size_t bitmap_bytes(int num_pages) { return (size_t)(((num_pages + 31) / 32 + kBlocks - 1) / kBlocks) * 4; }

}  // namespace

cudaError_t hswa_launch_pages_fork(const PagesForkParams& params, int num_sms, cudaStream_t s) {
  PagesForkParams p = params;
  p.second = (int64_t)p.rows_in * p.max_blocks + (int64_t)p.rows_out * p.out_max_blocks > kSmallTables;
  p.copied = p.num_pages > kSmallPool;
  if (p.copied) pages_copy_counts_kernel<<<4 * num_sms, kWideThreads, 0, s>>>(p.ref, p.ref_out, nullptr, reinterpret_cast<uint32_t*>(p.fresh), p.num_pages);
  const cudaError_t e = launch_cluster<pages_fork_kernel>(p, ((size_t)p.rows_in * 3 + (size_t)p.rows_out * 4) * 4 + bitmap_bytes(p.num_pages), s);
  return e != cudaSuccess || !p.second ? e : launch_wide(pages_fork_apply_kernel, p, num_sms, s);
}
cudaError_t hswa_launch_pages_compact(const PagesCompactParams& params, int num_sms, cudaStream_t s) {
  PagesCompactParams p = params;
  p.second = (int64_t)p.rows * p.max_blocks > kSmallTables;
  p.copied = p.num_pages > kSmallPool;
  if (p.copied) pages_copy_counts_kernel<<<4 * num_sms, kWideThreads, 0, s>>>(p.ref, p.ref_out, p.page_map, reinterpret_cast<uint32_t*>(p.page_map), p.num_pages);
  const cudaError_t e = launch_cluster<pages_compact_kernel>(p, 2 * bitmap_bytes(p.num_pages), s);
  return e != cudaSuccess || !p.second ? e : launch_wide(pages_compact_apply_kernel, p, num_sms, s);
}
cudaError_t hswa_launch_pages_copy(const PagesCopyParams& p, cudaStream_t s) {
  const int chunks = (int)((p.page_bytes + kCopyBytes - 1) / kCopyBytes);
  pages_copy_kernel<<<dim3((unsigned)((int64_t)p.pairs * chunks), p.n_pools, 1), kCopyThreads, 0, s>>>(p, chunks);
  return cudaGetLastError();
}
