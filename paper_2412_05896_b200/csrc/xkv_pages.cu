// Pages of the caches copied, shared, given back and moved (bookkeeping of the reduced caches whose sizes differ per layer,
// Sec. IV-A: the same step for the caches of all layers).
//
//   xkv_fork_caches    cache (l, b) becomes cache (l, parent[b]) cut to keep[l][b] rows: forks share whole pages, partly filled
//                      last pages are copied where others hold them, pages that nobody holds go back to the free list
//   xkv_compact_pages  pages in use become pages 0 .. n_live-1 of the pool
//   xkv_copy_pages     pages of one pool copied into another
//
// The first two are a plan and a copy of rows or pages by the whole GPU whose CTAs are in place when the plan ends.  A plan of few
// caches and pages is one CTA's, with the counters in its shared memory, in one launch with the copy (a cluster of eight; 96 caches
// 14 us, 8 caches compacted 6.7); of larger ones all SMs count the holders and write tables and rows, and what has an order (pages off the
// list and back to it) is decided in between by a cluster with barriers between its phases (1024 caches of 32 layers forked and ended
// 46 us, of which tables and rows 20).
// A plan is bound by latency: dependent loads, and code that runs once out of a cold instruction cache, which is why its
// loops are not unrolled further; the copy by HBM (527 MB 83 us = 0.97 of the measured copy rate).
#include <algorithm>
#include <atomic>

#include "common.cuh"
#include "e4m3.cuh"
#include "ops.h"

namespace xkv {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kMaxCluster = 8;        // the largest portable cluster
constexpr int kCopyThreads = 256;
constexpr int kPiece = 4096;          // bytes of K or V a warp copies at a time: eight 16-byte loads a lane in flight

// ---------------------------------------------------------------------------------------------
// Copies of rows
// ---------------------------------------------------------------------------------------------
struct RowCopy {
  int32_t src, dst, rows;             // pages, and how many of the first rows of every KV head; rows 0: nothing
};

struct Pool {
  uint8_t* k_pages;
  uint8_t* v_pages;
  float* k_scales;
  float* v_scales;
};

struct CopyParams {
  Pool from, to;
  int32_t n_kv_heads, page_size, row_bytes, pieces;   // pieces: of a page's rows of one head
  int32_t scale_rows;                 // rows a scale stands for, 0: no scales
};

// One warp: the rows of one head, of K (part < n_kv_heads) or of V, from piece `piece` on, every `step`-th.
__device__ __forceinline__ void copy_head(const CopyParams& p, const RowCopy& c, int part, int piece, int step) {
  const int lane = threadIdx.x & 31;
  const bool is_v = part >= p.n_kv_heads;
  const int h = is_v ? part - p.n_kv_heads : part, bytes = c.rows * p.row_bytes;
  const size_t from = (size_t)c.src * p.n_kv_heads + h, to = (size_t)c.dst * p.n_kv_heads + h;
  const size_t page_bytes = (size_t)p.page_size * p.row_bytes;
  const uint8_t* s = (is_v ? p.from.v_pages : p.from.k_pages) + from * page_bytes;
  uint8_t* d = (is_v ? p.to.v_pages : p.to.k_pages) + to * page_bytes;
  if (p.scale_rows > 0 && piece == 0) {
    const int n = (c.rows + p.scale_rows - 1) / p.scale_rows, per = p.page_size / p.scale_rows;
    const float* ss = (is_v ? p.from.v_scales : p.from.k_scales) + from * per;
    float* ds = (is_v ? p.to.v_scales : p.to.k_scales) + to * per;
    for (int i = lane; i < n; i += 32) ds[i] = ss[i];
  }
#pragma unroll 1
  for (int at = piece * kPiece; at < bytes; at += step * kPiece) {
    const uint4* s4 = reinterpret_cast<const uint4*>(s + at) + lane;
    uint4* d4 = reinterpret_cast<uint4*>(d + at) + lane;
    const int n = min(bytes - at, kPiece) / 16;
    uint4 v[kPiece / 512];
#pragma unroll
    for (int i = 0; i < kPiece / 512; ++i)
      if (i * 32 + lane < n) v[i] = __ldcs(s4 + i * 32);
#pragma unroll
    for (int i = 0; i < kPiece / 512; ++i)
      if (i * 32 + lane < n) __stcs(d4 + i * 32, v[i]);
  }
}

// Calls f(copy, part, piece, step) for this warp's share of n copies: a head's rows go to as many warps as a page has pieces,
// which take every step-th piece (whole pages) or all to one warp (the first rows of pages, often less than a piece).
template <typename F>
__device__ __forceinline__ void each_head(const CopyParams& p, int64_t n, bool whole, F f) {
  const int step = whole ? p.pieces : 1, per = 2 * p.n_kv_heads * step;
  const int64_t warp = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t n_warps = (int64_t)gridDim.x * (blockDim.x >> 5), end = n * per;
  if (end <= 0x7fffffffll - n_warps) {
    for (int u = (int)warp; u < (int)end; u += (int)n_warps) {
      const int c = u / per, rest = u - c * per;
      f(c, rest / step, rest % step, step);
    }
  } else {
    for (int64_t u = warp; u < end; u += n_warps) f(u / per, (int)(u % per) / step, (int)(u % per) % step, step);
  }
}

// The list that a plan has made: entries and their number in the workspace.
__device__ __forceinline__ void copy_rows(const CopyParams& p, const RowCopy* list, int n) {
  each_head(p, n, false, [&](int64_t i, int part, int piece, int step) {
    copy_head(p, {__ldcg(&list[i].src), __ldcg(&list[i].dst), __ldcg(&list[i].rows)}, part, piece, step);
  });
}

// Page ids that a caller gives.
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const CopyParams p, const int32_t* src, const int32_t* dst,
                                                                  int64_t n_copies, int32_t n_from, int32_t n_to,
                                                                  WorkspaceHeader* hdr) {
  each_head(p, n_copies, true, [&](int64_t i, int part, int piece, int step) {
    const RowCopy c = {__ldg(&src[i]), __ldg(&dst[i]), p.page_size};
    if (c.src < 0 || c.src >= n_from || c.dst < 0 || c.dst >= n_to) {
      if (part == 0 && piece == 0 && (threadIdx.x & 31) == 0) record_status(hdr, XKV_ERR_INVALID_ARG);
      return;
    }
    copy_head(p, c, part, piece, step);
  });
}

CopyParams copy_params(const xkv_dims* d, const xkv_cache* from, const xkv_cache* to) {
  CopyParams p;
  p.from = {static_cast<uint8_t*>(from->k_pages), static_cast<uint8_t*>(from->v_pages), from->k_scales, from->v_scales};
  p.to = {static_cast<uint8_t*>(to->k_pages), static_cast<uint8_t*>(to->v_pages), to->k_scales, to->v_scales};
  p.n_kv_heads = d->n_kv_heads;
  p.page_size = from->page_size;
  p.row_bytes = d->head_dim * (from->kv_format == XKV_KV_BF16 ? 2 : 1);
  p.pieces = (p.page_size * p.row_bytes + kPiece - 1) / kPiece;
  p.scale_rows = from->kv_format == XKV_KV_BF16 ? 0 : (from->kv_format == XKV_KV_INT8 ? 1 : kScaleBlock);
  return p;
}

// Whole pages: four waves of CTAs, which even out (2011 pages of 131 KB 83.1 us, one wave 87.1; 565 MB of a pool that is compacted 93.8 and
// 96.0, and 101.5 with stores that stay in L2); rows of a plan that is still to come: one, which is in place when it ends.
int copy_grid(const CopyParams& p, int64_t most_copies, bool whole) {
  const int64_t warps = most_copies * 2 * p.n_kv_heads * (whole ? p.pieces : 1);
  const int64_t ctas = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  return (int)std::max<int64_t>(1, std::min<int64_t>(ctas, (whole ? 32 : 8) * (int64_t)sm_count()));
}

// ---------------------------------------------------------------------------------------------
// Phases of a cluster
// ---------------------------------------------------------------------------------------------
// Every thread of the cluster; what its threads wrote before it, all of them see behind it.
__device__ __forceinline__ void phase() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// Exclusive prefix of x over the CTA's threads, and its sum.  s: kPlanWarps + 1 ints; every thread.
__device__ __forceinline__ int block_scan(int x, int* s, int* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();                    // s may still be read from the call before
  if (lane == 31) s[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const int w = s[lane];
    int wi = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xffffffffu, wi, o);
      if (lane >= o) wi += y;
    }
    s[lane] = wi - w;
    if (lane == 31) s[32] = wi;
  }
  __syncthreads();
  *total = s[32];
  return s[warp] + incl - x;
}

// This CTA's share of n things, in whole warps.
__device__ __forceinline__ void cta_run(int64_t n, int64_t* begin, int64_t* end) {
  const int64_t run = ((n + gridDim.x - 1) / gridDim.x + 31) / 32 * 32;
  *begin = min(n, run * (int64_t)blockIdx.x);
  *end = min(n, *begin + run);
}

// ---------------------------------------------------------------------------------------------
// Forks, cuts and frees
// ---------------------------------------------------------------------------------------------
struct ForkParams {
  int32_t* table;                     // [L][B][cols]
  int32_t* lens;                      // [L][B]
  const int32_t* parent;
  const int32_t* keep;
  int32_t keep_stride;
  int32_t* shares;
  int32_t* free_pages;
  int32_t n_free;
  int32_t* used;
  int32_t n_rows, batch, cols, page_size, n_pages;    // n_rows: caches, L * B
  WorkspaceHeader* hdr;
  int32_t* n_copies;                  // of the list
  int32_t* counts;                    // [2][kMaxCluster] copies and returned pages of the CTAs
  RowCopy* list;                      // [L * B]
  int4* rows;                         // [L * B] a ForkRow each
  int32_t* last;                      // [L * B] partly filled last page, -1: none
  int32_t* rank;                      // [L * B] place among the CTA's copies, -1: no copy
  // a bit a page: it may have lost its last holder, then: it has.  A call leaves it zero.  Bits that were there all the same (the workspace
  // served another pool or operator) do no harm: fork_decide looks at the counter of each, and a page with holders drops out.
  uint32_t* gone;
  int32_t* word_at;                   // bits before each of its words, within a CTA's share of them
  int32_t* fresh;                     // [L][B][cols] entries of caches that become forks
};

__device__ __forceinline__ bool in_pool(const ForkParams& p, int page) { return page >= 0 && page < p.n_pages; }

struct ForkRow {
  int32_t parent, rows, have, need;   // parent -1: freed; rows after the step; pages before and after it
};
__device__ __forceinline__ ForkRow as_row(int4 x) { return {x.x, x.y, x.z, x.w}; }

__device__ __forceinline__ int parent_of(const ForkParams& p, int b) {
  const int a = __ldcg(&p.parent[b]);
  return a >= -1 && a < p.batch ? a : b;
}

// What becomes of a cache; lengths as they were before the step.
__device__ __forceinline__ int4 fork_row(const ForkParams& p, int row) {
  const int l = row / p.batch, b = row - l * p.batch, most = p.cols * p.page_size;
  const int own = __ldcg(&p.lens[row]), k = p.keep != nullptr ? __ldcg(&p.keep[(size_t)l * p.keep_stride + b]) : -1;
  const int asked = __ldcg(&p.parent[b]), a = asked >= -1 && asked < p.batch ? asked : b;
  if (a != asked) record_status(p.hdr, XKV_ERR_INVALID_ARG);
  const int n = min(max(own, 0), most);
  int rows = a < 0 ? 0 : (a == b ? n : min(max(__ldcg(&p.lens[(size_t)l * p.batch + a]), 0), most));
  if (k >= 0) rows = min(rows, k);
  return make_int4(a, rows, (n + p.page_size - 1) / p.page_size, (rows + p.page_size - 1) / p.page_size);
}

// The page that a cache's partly filled last rows are in, as its parent's table has it; -1: none.
__device__ __forceinline__ int last_page(const ForkParams& p, int row, const ForkRow& r) {
  if (r.rows % p.page_size == 0) return -1;
  const int b = row % p.batch, e = __ldcg(&p.table[((size_t)(row - b) + r.parent) * p.cols + r.need - 1]);
  return in_pool(p, e) ? e : -1;
}

// A warp: holders that come and go, in whatever order (who is free shows at the end), and the entries that a fork gets.  No table
// changes yet: others read their parents' entries.
__device__ __forceinline__ void count_holders(const ForkParams& p, int row, const ForkRow& r) {
  const int lane = threadIdx.x & 31, b = row % p.batch;
  const int32_t* mine = p.table + (size_t)row * p.cols;
  const int32_t* theirs = p.table + ((size_t)(row - b) + max(r.parent, 0)) * p.cols;
  int32_t* fresh = p.fresh + (size_t)row * p.cols;
#pragma unroll 4
  for (int i = (r.parent == b ? r.need : 0) + lane; i < max(r.have, r.need); i += 32) {
    const bool had = i < r.have, gets = i < r.need;
    const int was = had ? __ldcg(&mine[i]) : -1, now = gets ? __ldcg(&theirs[i]) : -1;
    if (gets) fresh[i] = now;
    if ((had && !in_pool(p, was)) || (gets && !in_pool(p, now))) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    if (had && gets && was == now) continue;
    if (gets && in_pool(p, now)) atomicAdd(&p.shares[now], 1);
    // (a page that ends without a holder has had one taken at no others, whatever came between)
    if (had && in_pool(p, was) && atomicSub(&p.shares[was], 1) <= 0) atomicOr(&p.gone[was >> 5], 1u << (was & 31));
  }
}

// The whole cluster: pages for copies, lengths, and pages back to the list.  row_at(row): its ForkRow.
template <typename RowAt>
__device__ __forceinline__ void fork_decide(const ForkParams& p, RowAt row_at) {
  __shared__ int s_scan[kPlanWarps + 1];
  __shared__ int4 s_held[kPlanThreads];            // cache, its page, others that hold it
  __shared__ int s_copy[kPlanThreads];
  // ---- last pages that need a copy: those that others hold too, unless all holders are such last pages, of which one
  //      (the cache that stays, else the first) keeps it.  A thread a cache; a warp for each that others hold, which looks through its
  //      layer's caches (so this grows with their square: a fork of 512, 2048, 8192 caches in each of four layers and its end 53, 369,
  //      5125 us).
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int64_t row0, row1;
  cta_run(p.n_rows, &row0, &row1);
  // of a thread's first cache and first word, which are the only ones in most calls: kept in registers past the barriers
  const bool has = row0 + threadIdx.x < row1;
  const ForkRow first_row = has ? row_at((int)row0 + threadIdx.x) : ForkRow{0, 0, 0, 0};
  int first_last = -1, first_rank = -1;
  int copies = 0;
  for (int64_t base = row0; base < row1; base += kPlanThreads) {
    const int mine = (int)base + threadIdx.x;
    const int own = mine < row1 ? __ldcg(&p.last[mine]) : -1;
    const int own_others = own >= 0 ? __ldcg(&p.shares[own]) : 0;
    const bool held_by_others = own_others > 0;
    s_copy[threadIdx.x] = 0;
    int n_held, total;
    const int place = block_scan(held_by_others ? 1 : 0, s_scan, &n_held);
    if (held_by_others) s_held[place] = make_int4(mine, own, own_others, 0);
    __syncthreads();
#pragma unroll 2
    for (int i = warp; i < n_held; i += kPlanWarps) {
      const int4 h = s_held[i];
      const int row = h.x, page = h.y, others = h.z, b0 = row % p.batch;
      int n = 0, first = 0x7fffffff;
#pragma unroll 2
      for (int b = lane; b < p.batch; b += 32)
        if (__ldcg(&p.last[row - b0 + b]) == page) {
          ++n;
          first = min(first, b + (parent_of(p, b) == b ? 0 : p.batch));
        }
      n = __reduce_add_sync(0xffffffffu, n);
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0) s_copy[row - base] = !(n == others + 1 && (first == b0 || first == b0 + p.batch));
    }
    __syncthreads();
    const int copy = s_copy[threadIdx.x], before = block_scan(copy, s_scan, &total);
    if (base == row0) {
      first_last = own;
      first_rank = copy ? before : -1;
    } else if (mine < row1) {
      p.rank[mine] = copy ? copies + before : -1;
    }
    copies += total;
  }
  const int n_words = (p.n_pages + 31) / 32;
  int64_t word0, word1;
  cta_run(n_words, &word0, &word1);
  int back = 0, first_at = 0;
  for (int64_t w0 = word0 + warp; w0 < word1; w0 += 4 * kPlanWarps) {           // four words of a warp are asked for together
    uint32_t word[4];
    int holders[4];                   // beyond the first
#pragma unroll
    for (int u = 0; u < 4; ++u) word[u] = w0 + u * kPlanWarps < word1 ? __ldcg(&p.gone[w0 + u * kPlanWarps]) : 0u;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t page = (w0 + u * kPlanWarps) * 32 + lane;           // (the last word has bits behind the pool)
      holders[u] = ((word[u] >> lane) & 1u) != 0 && page < p.n_pages ? __ldcg(&p.shares[page]) : 0;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (holders[u] < -1) record_status(p.hdr, XKV_ERR_INVALID_ARG);          // dropped more often than it was held
      const uint32_t left = __ballot_sync(0xffffffffu, holders[u] < 0);
      if (lane == 0 && left != word[u]) p.gone[w0 + u * kPlanWarps] = left;
    }
  }
  __syncthreads();
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    int total;
    const int before = block_scan(w < word1 ? __popc(__ldcg(&p.gone[w])) : 0, s_scan, &total);
    if (base == word0) first_at = before;
    else if (w < word1) p.word_at[w] = back + before;
    back += total;
  }
  if (threadIdx.x == 0) {
    p.counts[blockIdx.x] = copies;
    p.counts[kMaxCluster + blockIdx.x] = back;
  }
  const int used = min(max(__ldcg(p.used), 0), p.n_free);
  phase();
  // ---- pages for the copies, from the list as it was; lengths (read for the last time before the phases here)
  int copies_before = 0, back_before = 0, all_copies = 0, all_back = 0;
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const int c = __ldcg(&p.counts[i]), r = __ldcg(&p.counts[kMaxCluster + i]);
    if (i < (int)blockIdx.x) copies_before += c, back_before += r;
    all_copies += c, all_back += r;
  }
  for (int64_t base = row0; base < row1; base += kPlanThreads) {
    const int row = (int)base + threadIdx.x;
    if (row >= row1) continue;
    const bool kept = base == row0;
    const ForkRow r = kept ? first_row : row_at(row);
    const int rank = kept ? first_rank : p.rank[row];
    int rows = r.rows;
    if (rank >= 0) {
      const int i = copies_before + rank, page = kept ? first_last : p.last[row];
      const int to = i < p.n_free - used ? __ldcg(&p.free_pages[used + i]) : -1;
      atomicSub(&p.shares[page], 1);
      RowCopy c = {page, to, r.rows % p.page_size};
      if (in_pool(p, to)) {
        (r.parent == row % p.batch ? p.table : p.fresh)[(size_t)row * p.cols + r.need - 1] = to;
      } else {                        // no page: only whole pages stay
        record_status(p.hdr, i < p.n_free - used ? XKV_ERR_INVALID_ARG : XKV_ERR_CAPACITY);
        c = {0, 0, 0};
        rows -= rows % p.page_size;
      }
      p.list[i] = c;
    }
    p.lens[row] = rows;
  }
  if (all_copies > 0 && all_back > 0) phase();       // (the list is read above where it is written below; the same for all CTAs)
  // ---- pages back to the list, in ascending order
  const int taken = min(all_copies, p.n_free - used);
  const int top = used + taken - all_back;
  for (int64_t w = word0 + threadIdx.x; w < word1; w += kPlanThreads) {
    uint32_t bits = __ldcg(&p.gone[w]);
    if (bits == 0) continue;
    p.gone[w] = 0u;
    for (int at = top + back_before + (w < word0 + kPlanThreads ? first_at : p.word_at[w]); bits != 0; bits &= bits - 1, ++at) {
      const int page = (int)w * 32 + __ffs(bits) - 1;
      p.shares[page] = 0;
      if (at >= 0) p.free_pages[at] = page;
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (top < 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);    // more came back than were handed out
    *p.used = max(top, 0);
    *p.n_copies = all_copies;
  }
}

// All of a step in one launch: the first CTA of a cluster plans with the pool's counters and the caches' new entries in its shared
// memory (three round trips to global memory: lengths and counters, entries, free pages), then all of them copy the rows.
struct SmallFork {                    // its shared memory, in ints
  int32_t holders, fresh, lens, last, copy, words, rows, total;
};
__host__ __device__ inline SmallFork small_fork(int n_rows, int cols, int n_pages) {
  SmallFork s;
  int at = 0;
  s.rows = at;    at += 4 * n_rows;
  s.holders = at; at += n_pages;                     // beyond the first
  s.fresh = at;   at += n_rows * cols;
  s.lens = at;    at += n_rows;
  s.last = at;    at += n_rows;
  s.copy = at;    at += n_rows;                      // page of the copy, -1: none, -2: wanted, -3: there was no page
  s.words = at;   at += (n_pages + 31) / 32;         // a bit a page: dropped by a cache
  s.total = at;
  return s;
}

__global__ void __launch_bounds__(kPlanThreads, 1) fork_small_kernel(const ForkParams p, const CopyParams c) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  extern __shared__ __align__(16) int32_t s_mem[];           // (rows are read as int4)
  __shared__ int s_scan[kPlanWarps + 1];
  __shared__ int s_busy[kPlanThreads];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (blockIdx.x == 0) {
    const SmallFork at = small_fork(p.n_rows, p.cols, p.n_pages);
    int4* s_rows = reinterpret_cast<int4*>(s_mem + at.rows);
    int *s_holders = s_mem + at.holders, *s_fresh = s_mem + at.fresh, *s_lens = s_mem + at.lens, *s_last = s_mem + at.last;
    int* s_copy = s_mem + at.copy;
    uint32_t* s_words = reinterpret_cast<uint32_t*>(s_mem + at.words);
    const int n_words = (p.n_pages + 31) / 32, most = p.cols * p.page_size;
    const int used = min(max(__ldcg(p.used), 0), p.n_free);
    for (int i = tid; i < p.n_rows; i += kPlanThreads) s_lens[i] = min(max(__ldcg(&p.lens[i]), 0), most);
#pragma unroll 4
    for (int i = tid; i < p.n_pages; i += kPlanThreads) s_holders[i] = __ldcg(&p.shares[i]);
    for (int i = tid; i < n_words; i += kPlanThreads) s_words[i] = 0u;
    __syncthreads();
    for (int row = tid; row < p.n_rows; row += kPlanThreads) {
      const int l = row / p.batch, b = row - l * p.batch, asked = __ldcg(&p.parent[b]);
      const int a = asked >= -1 && asked < p.batch ? asked : b;
      if (a != asked) record_status(p.hdr, XKV_ERR_INVALID_ARG);
      int rows = a < 0 ? 0 : s_lens[row - b + a];
      if (p.keep != nullptr) {
        const int k = __ldcg(&p.keep[(size_t)l * p.keep_stride + b]);
        if (k >= 0) rows = min(rows, k);
      }
      const ForkRow r = {a, rows, (s_lens[row] + p.page_size - 1) / p.page_size, (rows + p.page_size - 1) / p.page_size};
      s_rows[row] = make_int4(r.parent, r.rows, r.have, r.need);
      s_last[row] = last_page(p, row, r);
      s_copy[row] = -1;
    }
    __syncthreads();
    // ---- holders that come and go (a page is free if none is left at the end, in whatever order), of caches that change
    int n_busy;
    {
      const ForkRow r = tid < p.n_rows ? as_row(s_rows[tid]) : ForkRow{0, 0, 0, 0};
      const bool busy = tid < p.n_rows && (r.parent != tid % p.batch || r.have > r.need);
      const int place = block_scan(busy ? 1 : 0, s_scan, &n_busy);
      if (busy) s_busy[place] = tid;
      __syncthreads();
    }
    for (int i_row = warp; i_row < n_busy; i_row += kPlanWarps) {
      const int row = s_busy[i_row], b = row % p.batch;
      const ForkRow r = as_row(s_rows[row]);
      const int32_t* mine = p.table + (size_t)row * p.cols;
      const int32_t* theirs = p.table + ((size_t)(row - b) + max(r.parent, 0)) * p.cols;
#pragma unroll 4
      for (int i = (r.parent == b ? r.need : 0) + lane; i < max(r.have, r.need); i += 32) {
        const int was = i < r.have ? __ldcg(&mine[i]) : -1, now = i < r.need ? __ldcg(&theirs[i]) : -1;
        if (i < r.need) s_fresh[row * p.cols + i] = now;
        if ((i < r.have && !in_pool(p, was)) || (i < r.need && !in_pool(p, now))) record_status(p.hdr, XKV_ERR_INVALID_ARG);
        if (i < r.have && i < r.need && was == now) continue;
        if (i < r.need && in_pool(p, now)) atomicAdd(&s_holders[now], 1);
        if (i < r.have && in_pool(p, was)) {
          atomicSub(&s_holders[was], 1);
          atomicOr(&s_words[was >> 5], 1u << (was & 31));
        }
      }
    }
    __syncthreads();
    // ---- tables; last pages that others hold too (see fork_decide)
    for (int row = warp; row < p.n_rows; row += kPlanWarps) {
      const ForkRow r = as_row(s_rows[row]);
      const int b0 = row % p.batch, page = s_last[row];
      if (r.parent != b0)
        for (int i = lane; i < r.need; i += 32) p.table[(size_t)row * p.cols + i] = s_fresh[row * p.cols + i];
      const int others = page >= 0 ? s_holders[page] : 0;
      if (others <= 0) continue;
      int n = 0, first = 0x7fffffff;
      for (int b = lane; b < p.batch; b += 32)
        if (s_last[row - b0 + b] == page) {
          ++n;
          first = min(first, b + (s_rows[row - b0 + b].x == b ? 0 : p.batch));
        }
      n = __reduce_add_sync(0xffffffffu, n);
      first = __reduce_min_sync(0xffffffffu, first);
      if (lane == 0 && !(n == others + 1 && (first == b0 || first == b0 + p.batch))) s_copy[row] = -2;
    }
    __syncthreads();
    // ---- pages for the copies, from the list as it was
    int copies = 0;
    for (int base = 0; base < p.n_rows; base += kPlanThreads) {
      const int row = base + tid;
      const bool copy = row < p.n_rows && s_copy[row] == -2;
      int total;
      const int i = copies + block_scan(copy ? 1 : 0, s_scan, &total);
      copies += total;
      if (row >= p.n_rows) continue;
      const ForkRow r = as_row(s_rows[row]);
      int rows = r.rows;
      if (copy) {
        const int page = s_last[row], to = i < p.n_free - used ? __ldcg(&p.free_pages[used + i]) : -1;
        atomicSub(&s_holders[page], 1);
        RowCopy x = {page, to, r.rows % p.page_size};
        if (in_pool(p, to)) {
          p.table[(size_t)row * p.cols + r.need - 1] = to;
        } else {                      // no page: only whole pages stay
          record_status(p.hdr, i < p.n_free - used ? XKV_ERR_INVALID_ARG : XKV_ERR_CAPACITY);
          x = {0, 0, 0};
          rows -= rows % p.page_size;
        }
        p.list[i] = x;
      }
      p.lens[row] = rows;
    }
    // ---- pages back to the list, in ascending order, and the counters: a thread a page, a warp a word of the map
    __syncthreads();
    for (int base = 0; base < p.n_pages; base += kPlanThreads) {
      const int page = base + tid;
      const bool gone = page < p.n_pages && ((s_words[page >> 5] >> lane) & 1u) != 0 && s_holders[page] < 0;
      const uint32_t word = __ballot_sync(0xffffffffu, gone);
      if (lane == 0 && page < p.n_pages) s_words[page >> 5] = word;
      if (page < p.n_pages) {
        if (gone && s_holders[page] < -1) record_status(p.hdr, XKV_ERR_INVALID_ARG);   // dropped more often than it was held
        p.shares[page] = max(s_holders[page], 0);
      }
    }
    __syncthreads();
    int back;                         // (at most kPlanThreads words)
    const int before = block_scan(tid < n_words ? __popc(s_words[tid]) : 0, s_scan, &back);
    if (tid < n_words) s_busy[tid] = before;
    __syncthreads();
    const int top = used + min(copies, p.n_free - used) - back;
    for (int page = tid; page < p.n_pages; page += kPlanThreads) {
      const uint32_t word = s_words[page >> 5];
      const int at_list = top + s_busy[page >> 5] + __popc(word & ((1u << lane) - 1u));
      if (((word >> lane) & 1u) != 0 && at_list >= 0) p.free_pages[at_list] = page;
    }
    if (tid == 0) {
      if (top < 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);      // more came back than were handed out
      *p.used = max(top, 0);
      *p.n_copies = copies;
    }
  }
  phase();
  copy_rows(c, p.list, __ldcg(p.n_copies));
}

// The same in three launches, whose first and last take all SMs.
__global__ void __launch_bounds__(kCopyThreads) fork_count_kernel(const ForkParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int n_warps = gridDim.x * (kCopyThreads / 32);
  for (int row = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); row < p.n_rows; row += n_warps) {
    const int4 r = fork_row(p, row);
    if ((threadIdx.x & 31) == 0) {
      p.rows[row] = r;
      p.last[row] = last_page(p, row, as_row(r));
    }
    count_holders(p, row, as_row(r));
  }
}
__global__ void __launch_bounds__(kPlanThreads, 1) fork_decide_kernel(const ForkParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  fork_decide(p, [&](int row) { return as_row(__ldcg(&p.rows[row])); });
}
// Tables of the forks, then the copies.
__global__ void __launch_bounds__(kCopyThreads) fork_finish_kernel(const ForkParams p, const CopyParams c) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n_warps = gridDim.x * (kCopyThreads / 32);
  for (int row = blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); row < p.n_rows; row += n_warps) {
    const ForkRow r = as_row(__ldcg(&p.rows[row]));
    if (r.parent == row % p.batch) continue;
#pragma unroll 4
    for (int i = threadIdx.x & 31; i < r.need; i += 32) {
      const size_t at = (size_t)row * p.cols + i;
      p.table[at] = __ldcg(&p.fresh[at]);
    }
  }
  copy_rows(c, p.list, __ldcg(p.n_copies));
}

// ---------------------------------------------------------------------------------------------
// Compaction of the pool
// ---------------------------------------------------------------------------------------------
struct CompactParams {
  const int32_t* before;              // tables [L][B][cols]
  int32_t* table;
  const int32_t* lens;
  const int32_t* shares_before;
  int32_t* shares;
  int32_t* free_pages;
  int32_t* used;
  int32_t n_rows, cols, page_size, n_pages;           // n_rows: caches, L * B
  WorkspaceHeader* hdr;
  int32_t* n_live;                    // pages in use, and those of them from n_live on
  int32_t* n_moved;
  int32_t* counts;                    // [kMaxCluster] pages in use of the CTAs' words
  uint32_t* live;                     // a bit a page: in use
  int32_t* word_at;                   // pages in use before each of its words
  RowCopy* list;                      // [n_pages] src and dst of the pages that move, in ascending order
  int32_t* place;                     // [n_pages] of a page that moves: its place in the list
};

// Pages that cache `row` holds.
__device__ __forceinline__ int held(const CompactParams& p, int64_t row) {
  return (min(max(__ldcg(&p.lens[row]), 0), p.cols * p.page_size) + p.page_size - 1) / p.page_size;
}

// A thread: where page `page` goes.  bits: its word of `live`, at: pages in use before that word, low: pages in use below n_live.
__device__ __forceinline__ void place_page(const CompactParams& p, int page, uint32_t bits, int at, int n_live, int low) {
  const bool in_use = (bits >> (page & 31)) & 1u;
  const int rank = at + __popc(bits & ((1u << (page & 31)) - 1u));        // pages in use below it
  if (page < n_live) {
    if (!in_use) p.list[page - rank].dst = page;
    else if (p.shares != nullptr) p.shares[page] = p.shares_before[page];
  } else if (in_use) {
    p.list[rank - low].src = page;
    p.list[rank - low].rows = p.page_size;
    p.place[page] = rank - low;
  } else if (p.shares != nullptr) {
    p.shares[page] = 0;
  }
}

// Tables, counters of the pages that move, the list; then the pages.
__device__ __forceinline__ void compact_move(const CompactParams& p, const CopyParams& c, int n_live, int n_moved) {
  const int64_t tid = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, step = (int64_t)gridDim.x * blockDim.x;
  const int64_t n_entries = (int64_t)p.n_rows * p.cols;
  for (int64_t i = tid; i < n_entries; i += step) {
    const int e = p.before[i];
    int now = e;
    if (e >= n_live && e < p.n_pages) {
      const int64_t row = i / p.cols;
      if (i - row * p.cols < held(p, row)) now = __ldcg(&p.list[__ldcg(&p.place[e])].dst);
    }
    p.table[i] = now;
  }
  if (p.free_pages != nullptr)
    for (int64_t i = n_live + tid; i < p.n_pages; i += step) p.free_pages[i] = (int)i;
  if (p.shares != nullptr)
    for (int64_t i = tid; i < n_moved; i += step) {
      const int src = __ldcg(&p.list[i].src), others = p.shares_before[src];
      p.shares[src] = 0;
      p.shares[__ldcg(&p.list[i].dst)] = others;
    }
  each_head(c, n_moved, true, [&](int64_t i, int part, int piece, int n) {
    copy_head(c, {__ldcg(&p.list[i].src), __ldcg(&p.list[i].dst), c.page_size}, part, piece, n);
  });
}

// Pools of up to kSmallWords words of a bit a page: every CTA of the cluster finds all pages in use for itself, in its shared memory,
// and places its share of them.  kMove: the move, too.
constexpr int kSmallWords = kPlanThreads;
template <bool kMove>
__global__ void __launch_bounds__(kPlanThreads, 1) compact_small_kernel(const CompactParams p, const CopyParams c) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ int s_scan[kPlanWarps + 1];
  __shared__ uint32_t s_live[kSmallWords];
  __shared__ int s_at[kSmallWords];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_words = (p.n_pages + 31) / 32;
  s_live[tid] = 0u;
  __syncthreads();
  for (int row = warp; row < p.n_rows; row += kPlanWarps) {
    const int have = held(p, row);
#pragma unroll 4
    for (int i = lane; i < have; i += 32) {
      const int e = p.before[(size_t)row * p.cols + i];
      if (e >= 0 && e < p.n_pages) atomicOr(&s_live[e >> 5], 1u << (e & 31));
      else record_status(p.hdr, XKV_ERR_INVALID_ARG);
    }
  }
  __syncthreads();
  int n_live;
  s_at[tid] = block_scan(__popc(s_live[tid]), s_scan, &n_live);
  __syncthreads();
  int low = n_live;                   // pages in use below n_live
  if ((n_live >> 5) < n_words) low = s_at[n_live >> 5] + __popc(s_live[n_live >> 5] & ((1u << (n_live & 31)) - 1u));
  for (int page = blockIdx.x * kPlanThreads + tid; page < p.n_pages; page += gridDim.x * kPlanThreads)
    place_page(p, page, s_live[page >> 5], s_at[page >> 5], n_live, low);
  if (blockIdx.x == 0 && tid == 0) {
    *p.n_live = n_live;
    *p.n_moved = n_live - low;
    *p.used = n_live;
  }
  if constexpr (kMove) {
    phase();                          // (also: every CTA has read the tables)
    compact_move(p, c, n_live, n_live - low);
  }
}

// The same for any pool, by a map in the workspace: which pages are in use, how many before each of its words.
__global__ void __launch_bounds__(kPlanThreads, 1) compact_count_kernel(const CompactParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ int s_scan[kPlanWarps + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = gridDim.x * kPlanWarps, n_words = (p.n_pages + 31) / 32;
  // (the map is cleared here, not at a call's end: another pool's or operator's call may have written over it since)
  for (int w = blockIdx.x * kPlanThreads + threadIdx.x; w < n_words; w += gridDim.x * kPlanThreads) p.live[w] = 0u;
  phase();
  for (int row = blockIdx.x * kPlanWarps + warp; row < p.n_rows; row += n_warps) {
    const int have = held(p, row);
#pragma unroll 4
    for (int i = lane; i < have; i += 32) {
      const int e = p.before[(size_t)row * p.cols + i];
      if (e >= 0 && e < p.n_pages) atomicOr(&p.live[e >> 5], 1u << (e & 31));
      else record_status(p.hdr, XKV_ERR_INVALID_ARG);
    }
  }
  phase();
  int64_t word0, word1;
  cta_run(n_words, &word0, &word1);
  int mine = 0;
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    int total;
    const int before = block_scan(w < word1 ? __popc(__ldcg(&p.live[w])) : 0, s_scan, &total);
    if (w < word1) p.word_at[w] = mine + before;
    mine += total;
  }
  if (threadIdx.x == 0) p.counts[blockIdx.x] = mine;
  phase();
  int n_live = 0, before = 0;
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const int n = __ldcg(&p.counts[i]);
    if (i < (int)blockIdx.x) before += n;
    n_live += n;
  }
  for (int64_t w = word0 + threadIdx.x; w < word1; w += kPlanThreads) p.word_at[w] += before;
  phase();
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int low = n_live;                 // pages in use below n_live
    if ((n_live >> 5) < n_words)
      low = __ldcg(&p.word_at[n_live >> 5]) + __popc(__ldcg(&p.live[n_live >> 5]) & ((1u << (n_live & 31)) - 1u));
    *p.n_live = n_live;
    *p.n_moved = n_live - low;
    *p.used = n_live;
  }
}

// Where its pages go.
__global__ void __launch_bounds__(kCopyThreads) compact_place_kernel(const CompactParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const int n_live = __ldcg(p.n_live), low = n_live - __ldcg(p.n_moved);
  const int64_t step = (int64_t)gridDim.x * kCopyThreads;
  for (int64_t page = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x; page < p.n_pages; page += step)
    place_page(p, (int)page, __ldcg(&p.live[page >> 5]), __ldcg(&p.word_at[page >> 5]), n_live, low);
}

__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const CompactParams p, const CopyParams c) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  compact_move(p, c, __ldcg(p.n_live), __ldcg(p.n_moved));
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct Layout {
  size_t counts, list, a, b, rows, bits, words, fresh, total;
};

Layout fork_layout(int64_t n_rows, int cols, int64_t n_pages) {
  Layout L;
  size_t off = kHeaderBytes;
  L.counts = off; off = align_up(off + (8 + 2 * kMaxCluster) * 4, 256);
  L.bits = off;   off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.words = off;  off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.list = off;   off = align_up(off + (size_t)n_rows * sizeof(RowCopy), 256);
  L.a = off;      off = align_up(off + (size_t)n_rows * 4, 256);
  L.b = off;      off = align_up(off + (size_t)n_rows * 4, 256);
  L.rows = off;   off = align_up(off + (size_t)n_rows * sizeof(int4), 256);
  L.fresh = off;  off = align_up(off + (size_t)n_rows * cols * 4, 256);
  L.total = off;
  return L;
}

Layout compact_layout(int64_t n_pages) {
  Layout L = {};
  size_t off = kHeaderBytes;
  L.counts = off; off = align_up(off + (8 + kMaxCluster) * 4, 256);
  L.bits = off;   off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.words = off;  off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.list = off;   off = align_up(off + (size_t)n_pages * sizeof(RowCopy), 256);
  L.a = off;      off = align_up(off + (size_t)n_pages * 4, 256);
  L.total = off;
  return L;
}

// All launches here wait for the one before them on the device, so that their CTAs may be in place when it ends.  What it may still be
// writing then (lengths, parents, counts) is read by ordinary loads, not through the read-only path, which is for data that nobody
// writes while the kernel is there.
template <typename... Args>
xkv_status launch_after(void (*kernel)(Args...), int grid, int threads, bool cluster, cudaStream_t st, size_t smem,
                        Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.dynamicSmemBytes = smem;
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)grid;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster ? 2 : 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
    (void)cudaGetLastError();
    return XKV_ERR_CUDA;
  }
  count_launch();
  return check_launch();
}

// Table entries, and pages of a pool, up to which one CTA plans a step's forks.
constexpr int64_t kManyEntries = 16384;
static_assert(kManyEntries / 32 <= kPlanThreads, "a thread a word of the map");
constexpr int kSmallForkBytes = 4 * (2 * kManyEntries + kManyEntries / 32 + 7 * kPlanThreads);
// Bytes that a plan's cluster copies itself: a second launch takes the device 2 us and the host 4.
constexpr int64_t kFewBytes = 2 << 20;

}  // namespace

size_t fork_workspace_bytes(int n_layers, int batch, int max_pages_per_seq, int64_t n_pages) {
  return fork_layout((int64_t)n_layers * batch, max_pages_per_seq, n_pages).total;
}
size_t compact_workspace_bytes(int64_t n_pages) { return compact_layout(n_pages).total; }
size_t copy_workspace_bytes() { return kHeaderBytes; }

xkv_status fork_caches(const xkv_dims* d, const xkv_cache* c, const int32_t* parent, const int32_t* keep, int keep_stride,
                       int32_t* shares, int32_t* free_pages, int n_free, int32_t* pages_used, void* workspace,
                       cudaStream_t st) {
  const int64_t n_rows = (int64_t)c->n_layers * d->batch;
  const Layout L = fork_layout(n_rows, c->max_pages_per_seq, c->n_pages);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  ForkParams p;
  p.table = c->block_table;
  p.lens = c->seq_lens;
  p.parent = parent;
  p.keep = keep;
  p.keep_stride = keep_stride;
  p.shares = shares;
  p.free_pages = free_pages;
  p.n_free = n_free;
  p.used = pages_used;
  p.n_rows = (int32_t)n_rows;
  p.batch = d->batch;
  p.cols = c->max_pages_per_seq;
  p.page_size = c->page_size;
  p.n_pages = c->n_pages;
  p.hdr = reinterpret_cast<WorkspaceHeader*>(ws);
  p.n_copies = reinterpret_cast<int32_t*>(ws + L.counts);
  p.counts = p.n_copies + 8;
  p.list = reinterpret_cast<RowCopy*>(ws + L.list);
  p.last = reinterpret_cast<int32_t*>(ws + L.a);
  p.rank = reinterpret_cast<int32_t*>(ws + L.b);
  p.rows = reinterpret_cast<int4*>(ws + L.rows);
  p.gone = reinterpret_cast<uint32_t*>(ws + L.bits);
  p.word_at = reinterpret_cast<int32_t*>(ws + L.words);
  p.fresh = reinterpret_cast<int32_t*>(ws + L.fresh);
  const CopyParams cp = copy_params(d, c, c);
  xkv_status s;
  // Few bytes of last rows at most, and little enough for one CTA's shared memory.
  if (n_rows * p.cols <= kManyEntries && n_rows <= kPlanThreads && p.n_pages <= kManyEntries &&
      n_rows * 2 * cp.n_kv_heads * cp.page_size * cp.row_bytes <= kFewBytes) {
    static std::atomic<bool> done[64];   // idempotent set-up: two threads doing it twice is harmless
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return XKV_ERR_CUDA;
    if (!done[dev].load(std::memory_order_acquire)) {
      if (cudaFuncSetAttribute(fork_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmallForkBytes) != cudaSuccess) {
        (void)cudaGetLastError();
        return XKV_ERR_CUDA;
      }
      done[dev].store(true, std::memory_order_release);
    }
    return launch_after(fork_small_kernel, kMaxCluster, kPlanThreads, true, st,
                        4 * (size_t)small_fork((int)n_rows, p.cols, p.n_pages).total, p, cp);
  }
  const int grid = (int)std::min<int64_t>((n_rows + kCopyThreads / 32 - 1) / (kCopyThreads / 32), 8 * (int64_t)sm_count());
  s = launch_after(fork_count_kernel, grid, kCopyThreads, false, st, 0, p);
  if (s == XKV_OK) s = launch_after(fork_decide_kernel, kMaxCluster, kPlanThreads, true, st, 0, p);
  if (s != XKV_OK) return s;
  return launch_after(fork_finish_kernel, std::max(grid, copy_grid(cp, n_rows, false)), kCopyThreads, false, st, 0, p, cp);
}

xkv_status compact_pages(const xkv_dims* d, const xkv_cache* c, const int32_t* table_before, const int32_t* shares_before,
                         int32_t* shares, int32_t* free_pages, int32_t* pages_used, void* workspace, cudaStream_t st) {
  const int64_t n_rows = (int64_t)c->n_layers * d->batch;
  const Layout L = compact_layout(c->n_pages);
  uint8_t* ws = static_cast<uint8_t*>(workspace);
  CompactParams p;
  p.before = table_before;
  p.table = c->block_table;
  p.lens = c->seq_lens;
  p.shares_before = shares_before;
  p.shares = shares;
  p.free_pages = free_pages;
  p.used = pages_used;
  p.n_rows = (int32_t)n_rows;
  p.cols = c->max_pages_per_seq;
  p.page_size = c->page_size;
  p.n_pages = c->n_pages;
  p.hdr = reinterpret_cast<WorkspaceHeader*>(ws);
  p.n_live = reinterpret_cast<int32_t*>(ws + L.counts);
  p.n_moved = p.n_live + 1;
  p.counts = p.n_live + 8;
  p.live = reinterpret_cast<uint32_t*>(ws + L.bits);
  p.word_at = reinterpret_cast<int32_t*>(ws + L.words);
  p.list = reinterpret_cast<RowCopy*>(ws + L.list);
  p.place = reinterpret_cast<int32_t*>(ws + L.a);
  const CopyParams cp = copy_params(d, c, c);
  xkv_status s;
  if (p.n_pages <= 32 * kSmallWords && n_rows * p.cols <= 4 * kManyEntries) {
    if ((int64_t)p.n_pages * 2 * cp.n_kv_heads * cp.page_size * cp.row_bytes <= kFewBytes)
      return launch_after(compact_small_kernel<true>, kMaxCluster, kPlanThreads, true, st, 0, p, cp);
    s = launch_after(compact_small_kernel<false>, kMaxCluster, kPlanThreads, true, st, 0, p, cp);
  } else {
    s = launch_after(compact_count_kernel, kMaxCluster, kPlanThreads, true, st, 0, p);
    const int64_t ctas = (p.n_pages + kCopyThreads - 1) / kCopyThreads;
    if (s == XKV_OK)
      s = launch_after(compact_place_kernel, (int)std::min<int64_t>(ctas, 8 * (int64_t)sm_count()), kCopyThreads, false, st, 0, p);
  }
  if (s != XKV_OK) return s;
  const int64_t entries = (n_rows * p.cols + 31) / 32;
  const int grid = std::max(copy_grid(cp, std::min<int64_t>(c->n_pages, n_rows * p.cols), true),
                            (int)std::min<int64_t>(entries / (kCopyThreads / 32), sm_count()));
  return launch_after(compact_move_kernel, grid, kCopyThreads, false, st, 0, p, cp);
}

xkv_status copy_pages(const xkv_dims* d, const xkv_cache* from, const int32_t* src, const xkv_cache* to, const int32_t* dst,
                      int64_t n_copies, void* workspace, cudaStream_t st) {
  const CopyParams p = copy_params(d, from, to);
  copy_pages_kernel<<<copy_grid(p, n_copies, true), kCopyThreads, 0, st>>>(p, src, dst, n_copies, from->n_pages, to->n_pages,
                                                                     static_cast<WorkspaceHeader*>(workspace));
  count_launch();
  return check_launch();
}

}  // namespace xkv
