// Pages of the caches copied, shared, given back and moved (bookkeeping of the reduced caches whose sizes differ per layer,
// Sec. IV-A: the same step for the caches of all layers).
//
//   xkv_fork_caches    cache (l, b) becomes cache (l, parent[b]) cut to keep[l][b] rows: forks share whole pages, partly filled
//                      last pages are copied where others hold them, pages that nobody holds go back to the free list
//   xkv_compact_pages  pages in use become pages 0 .. n_live-1 of the pool
//   xkv_copy_pages     pages of one pool copied into another
//
// The first two are a plan, one thread-block cluster whose phases are separated by cluster barriers (a grid of separate
// launches would pay a launch a phase), and a copy of rows or pages by the whole GPU whose CTAs are in place when the plan
// ends.  The plan is bound by latency: dependent loads of lengths, table entries and counters; the copy by HBM.
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

// One warp: piece `unit` of a list of row copies, numbered copy by copy, K before V, head by head.
__device__ __forceinline__ void copy_piece(const CopyParams& p, const RowCopy& c, int part) {
  const int lane = threadIdx.x & 31;
  const int piece = part % p.pieces, rest = part / p.pieces;
  const int h = rest % p.n_kv_heads, kv = rest / p.n_kv_heads;
  const int bytes = c.rows * p.row_bytes - piece * kPiece;
  if (bytes <= 0) return;
  const size_t from = (size_t)c.src * p.n_kv_heads + h, to = (size_t)c.dst * p.n_kv_heads + h;
  const size_t page_bytes = (size_t)p.page_size * p.row_bytes;
  const uint4* s = reinterpret_cast<const uint4*>((kv ? p.from.v_pages : p.from.k_pages) + from * page_bytes + (size_t)piece * kPiece);
  uint4* d = reinterpret_cast<uint4*>((kv ? p.to.v_pages : p.to.k_pages) + to * page_bytes + (size_t)piece * kPiece);
  const int n = min(bytes, kPiece) / 16;
  uint4 v[kPiece / 512];
#pragma unroll
  for (int i = 0; i < kPiece / 512; ++i)
    if (i * 32 + lane < n) v[i] = __ldcs(s + i * 32 + lane);
  float sc[8];
  const int n_scales = piece == 0 && p.scale_rows > 0 ? (c.rows + p.scale_rows - 1) / p.scale_rows : 0;
  const int page_scales = p.scale_rows > 0 ? p.page_size / p.scale_rows : 0;
#pragma unroll
  for (int i = 0; i < 8; ++i)         // a page has at most 256 rows
    if (i * 32 + lane < n_scales) sc[i] = (kv ? p.from.v_scales : p.from.k_scales)[from * page_scales + i * 32 + lane];
#pragma unroll
  for (int i = 0; i < kPiece / 512; ++i)
    if (i * 32 + lane < n) d[i * 32 + lane] = v[i];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (i * 32 + lane < n_scales) (kv ? p.to.v_scales : p.to.k_scales)[to * page_scales + i * 32 + lane] = sc[i];
}

// The list that a plan has made: entries and their number in the workspace.
__global__ void __launch_bounds__(kCopyThreads) copy_rows_kernel(const CopyParams p, const RowCopy* list, const int32_t* n_list) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int64_t per = 2 * (int64_t)p.n_kv_heads * p.pieces, n = __ldcg(n_list) * per;
  const int64_t step = (int64_t)gridDim.x * (kCopyThreads / 32);
  for (int64_t u = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); u < n; u += step) {
    const RowCopy c = {__ldcg(&list[u / per].src), __ldcg(&list[u / per].dst), __ldcg(&list[u / per].rows)};
    copy_piece(p, c, (int)(u % per));
  }
}

// Page ids that a caller gives.
__global__ void __launch_bounds__(kCopyThreads) copy_pages_kernel(const CopyParams p, const int32_t* src, const int32_t* dst,
                                                                  int64_t n_copies, int32_t n_from, int32_t n_to,
                                                                  WorkspaceHeader* hdr) {
  const int64_t per = 2 * (int64_t)p.n_kv_heads * p.pieces, n = n_copies * per;
  const int64_t step = (int64_t)gridDim.x * (kCopyThreads / 32);
  for (int64_t u = (int64_t)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); u < n; u += step) {
    const RowCopy c = {__ldg(&src[u / per]), __ldg(&dst[u / per]), p.page_size};
    if (c.src < 0 || c.src >= n_from || c.dst < 0 || c.dst >= n_to) {
      if (u % per == 0 && (threadIdx.x & 31) == 0) record_status(hdr, XKV_ERR_INVALID_ARG);
      continue;
    }
    copy_piece(p, c, (int)(u % per));
  }
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

int copy_grid(const CopyParams& p, int64_t most_copies) {
  const int64_t warps = most_copies * 2 * p.n_kv_heads * p.pieces;
  const int64_t ctas = (warps + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
  return (int)std::max<int64_t>(1, std::min<int64_t>(ctas, 8 * (int64_t)sm_count()));
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
  int32_t n_layers, batch, cols, page_size, n_pages;
  WorkspaceHeader* hdr;
  int32_t* n_copies;                  // of the list
  int32_t* counts;                    // [2][kMaxCluster] copies and returned pages of the CTAs
  RowCopy* list;                      // [L * B]
  int32_t* last;                      // [L * B] partly filled last page, -1: none
  int32_t* rank;                      // [L * B] place among the CTA's copies, -1: no copy
  uint32_t* gone;                     // a bit a page: nobody holds it any more; zero between calls
  int32_t* fresh;                     // [L][B][cols] entries of caches that become forks
};

__device__ __forceinline__ bool in_pool(const ForkParams& p, int page) { return page >= 0 && page < p.n_pages; }

struct ForkRow {
  int32_t parent, rows, have, need;   // parent -1: freed; rows after the step; pages before and after it
};

__device__ __forceinline__ int parent_of(const ForkParams& p, int b) {
  const int a = __ldg(&p.parent[b]);
  return a >= -1 && a < p.batch ? a : b;
}

// What becomes of cache (l, b); lengths as they were before the step.
__device__ __forceinline__ ForkRow fork_row(const ForkParams& p, int l, int b) {
  const int most = p.cols * p.page_size;
  ForkRow r;
  r.parent = parent_of(p, b);
  const int n = min(max(__ldcg(&p.lens[(size_t)l * p.batch + b]), 0), most);
  r.rows = r.parent < 0 ? 0 : (r.parent == b ? n : min(max(__ldcg(&p.lens[(size_t)l * p.batch + r.parent]), 0), most));
  if (p.keep != nullptr) {
    const int k = __ldg(&p.keep[(size_t)l * p.keep_stride + b]);
    if (k >= 0) r.rows = min(r.rows, k);
  }
  r.have = (n + p.page_size - 1) / p.page_size;
  r.need = (r.rows + p.page_size - 1) / p.page_size;
  return r;
}

__global__ void __launch_bounds__(kPlanThreads, 1) fork_kernel(const ForkParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ int s_scan[kPlanWarps + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_rows = p.n_layers * p.batch, n_warps = gridDim.x * kPlanWarps, w0 = blockIdx.x * kPlanWarps + warp;

  // ---- holders to come are counted first, so that no page seems to be free in between; the parents' entries are read
  //      before any table changes
  for (int row = w0; row < n_rows; row += n_warps) {
    const int l = row / p.batch, b = row % p.batch;
    const ForkRow r = fork_row(p, l, b);
    const int32_t* mine = p.table + (size_t)row * p.cols;
    const int32_t* theirs = p.table + ((size_t)l * p.batch + max(r.parent, 0)) * p.cols;
    int32_t* fresh = p.fresh + (size_t)row * p.cols;
    if (r.parent != b && lane == 0 && __ldg(&p.parent[b]) != r.parent) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    if (r.parent == b && lane == 0 && __ldg(&p.parent[b]) != b) record_status(p.hdr, XKV_ERR_INVALID_ARG);
    if (r.parent != b) {
      for (int i = lane; i < r.need; i += 32) {
        const int e = __ldcg(&theirs[i]);
        fresh[i] = e;
        if (in_pool(p, e)) {
          if (i >= r.have || __ldcg(&mine[i]) != e) atomicAdd(&p.shares[e], 1);
        } else {
          record_status(p.hdr, XKV_ERR_INVALID_ARG);
        }
      }
    }
    if (lane == 0) {
      const int e = r.rows % p.page_size != 0 ? __ldcg(&theirs[r.need - 1]) : -1;
      p.last[row] = in_pool(p, e) ? e : -1;
    }
  }
  // lengths are read again below, and change only behind the next barrier
  phase();
  // ---- entries that go, tables
  for (int row = w0; row < n_rows; row += n_warps) {
    const int l = row / p.batch, b = row % p.batch;
    const ForkRow r = fork_row(p, l, b);
    int32_t* mine = p.table + (size_t)row * p.cols;
    const int32_t* fresh = p.fresh + (size_t)row * p.cols;
    for (int i = (r.parent == b ? r.need : 0) + lane; i < max(r.have, r.need); i += 32) {
      const int now = i < r.need ? __ldcg(&fresh[i]) : -1;
      if (i < r.have) {
        const int was = __ldcg(&mine[i]);
        if (i < r.need && was == now) continue;
        if (in_pool(p, was)) {
          const int others = atomicSub(&p.shares[was], 1);
          if (others == 0) atomicOr(&p.gone[was >> 5], 1u << (was & 31));
          if (others < 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);
        } else {
          record_status(p.hdr, XKV_ERR_INVALID_ARG);
        }
      }
      if (i < r.need) mine[i] = now;
    }
  }
  phase();
  // ---- last pages that need a copy: those that others hold too, unless all holders are such last pages, of which one
  //      (the cache that stays, else the first) keeps it
  int64_t row0, row1;
  cta_run(n_rows, &row0, &row1);
  int copies = 0;
  for (int64_t base = row0; base < row1; base += kPlanThreads) {
    const int row = (int)base + threadIdx.x;
    const int page = row < row1 ? __ldcg(&p.last[row]) : -1;
    const int others = page >= 0 ? __ldcg(&p.shares[page]) : 0;
    bool copy = false;
    unsigned asked = __ballot_sync(0xffffffffu, others > 0);
    while (asked != 0) {
      const int src = __ffs(asked) - 1;
      asked &= asked - 1;
      const int q = __shfl_sync(0xffffffffu, page, src), at = __shfl_sync(0xffffffffu, row, src);
      const int n_others = __shfl_sync(0xffffffffu, others, src);
      const int l0 = at / p.batch * p.batch;
      int n = 0, first = 0x7fffffff;
      for (int b = lane; b < p.batch; b += 32)
        if (__ldcg(&p.last[l0 + b]) == q) {
          ++n;
          first = min(first, b + (parent_of(p, b) == b ? 0 : p.batch));
        }
      n = __reduce_add_sync(0xffffffffu, n);
      first = __reduce_min_sync(0xffffffffu, first);
      const int b = at - l0, key = b + (parent_of(p, b) == b ? 0 : p.batch);
      if (lane == src) copy = !(n == n_others + 1 && key == first);
    }
    int total;
    const int before = block_scan(copy ? 1 : 0, s_scan, &total);
    if (row < row1) p.rank[row] = copy ? copies + before : -1;
    copies += total;
  }
  const int n_words = (p.n_pages + 31) / 32;
  int64_t word0, word1;
  cta_run(n_words, &word0, &word1);
  int back = 0;
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    int total;
    block_scan(w < word1 ? __popc(__ldcg(&p.gone[w])) : 0, s_scan, &total);
    back += total;
  }
  if (threadIdx.x == 0) {
    p.counts[blockIdx.x] = copies;
    p.counts[kMaxCluster + blockIdx.x] = back;
  }
  phase();
  // ---- pages for the copies, from the list as it was
  int copies_before = 0, back_before = 0, all_copies = 0, all_back = 0;
  for (int i = 0; i < (int)gridDim.x; ++i) {
    const int c = __ldcg(&p.counts[i]), r = __ldcg(&p.counts[kMaxCluster + i]);
    if (i < (int)blockIdx.x) copies_before += c, back_before += r;
    all_copies += c, all_back += r;
  }
  const int used = min(max(__ldcg(p.used), 0), p.n_free);
  for (int64_t base = row0; base < row1; base += kPlanThreads) {
    const int row = (int)base + threadIdx.x;
    if (row >= row1) continue;
    const ForkRow r = fork_row(p, row / p.batch, row % p.batch);
    const int rank = p.rank[row];
    if (rank < 0) continue;
    const int i = copies_before + rank, page = p.last[row];
    const int to = i < p.n_free - used ? __ldcg(&p.free_pages[used + i]) : -1;
    atomicSub(&p.shares[page], 1);
    RowCopy c = {page, to, r.rows % p.page_size};
    if (in_pool(p, to)) {
      p.table[(size_t)row * p.cols + r.need - 1] = to;
    } else {                          // no page: only whole pages stay (see below)
      record_status(p.hdr, i < p.n_free - used ? XKV_ERR_INVALID_ARG : XKV_ERR_CAPACITY);
      c = {0, 0, 0};
      p.rank[row] = -2;
    }
    p.list[i] = c;
  }
  phase();
  // ---- lengths, and pages back to the list in ascending order
  for (int row = blockIdx.x * kPlanThreads + threadIdx.x; row < n_rows; row += gridDim.x * kPlanThreads) {
    // (a cache's own length is read by its forks above)
    const ForkRow r = fork_row(p, row / p.batch, row % p.batch);
    p.last[row] = __ldcg(&p.rank[row]) == -2 ? r.rows / p.page_size * p.page_size : r.rows;
  }
  const int taken = min(all_copies, p.n_free - used);
  const int top = used + taken - all_back;
  back = back_before;
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    uint32_t bits = w < word1 ? __ldcg(&p.gone[w]) : 0u;
    int total;
    int at = top + back + block_scan(__popc(bits), s_scan, &total);
    if (bits != 0) p.gone[w] = 0u;
    for (; bits != 0; bits &= bits - 1, ++at) {
      const int page = (int)w * 32 + __ffs(bits) - 1;
      p.shares[page] = 0;
      if (at >= 0) p.free_pages[at] = page;
    }
    back += total;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    if (top < 0) record_status(p.hdr, XKV_ERR_INVALID_ARG);    // more came back than were handed out
    *p.used = max(top, 0);
    *p.n_copies = all_copies;
  }
  phase();
  for (int row = blockIdx.x * kPlanThreads + threadIdx.x; row < n_rows; row += gridDim.x * kPlanThreads)
    p.lens[row] = __ldcg(&p.last[row]);
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
  int32_t n_layers, batch, cols, page_size, n_pages;
  WorkspaceHeader* hdr;
  int32_t* n_live;
  int32_t* n_moved;
  int32_t* counts;                    // [3][kMaxCluster] pages in use, gaps, pages that move, of the CTAs
  uint32_t* live;                     // a bit a page: in use; zero between calls
  RowCopy* list;                      // [n_pages] src and dst of the pages that move, in ascending order
  int32_t* place;                     // [n_pages] of a page that moves: its place in the list
};

__global__ void __launch_bounds__(kPlanThreads, 1) compact_kernel(const CompactParams p) {
  asm volatile("griddepcontrol.launch_dependents;");
  __shared__ int s_scan[kPlanWarps + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int n_rows = p.n_layers * p.batch, n_warps = gridDim.x * kPlanWarps;
  for (int row = blockIdx.x * kPlanWarps + warp; row < n_rows; row += n_warps) {
    const int have = (min(max(__ldg(&p.lens[row]), 0), p.cols * p.page_size) + p.page_size - 1) / p.page_size;
    for (int i = lane; i < have; i += 32) {
      const int e = p.before[(size_t)row * p.cols + i];
      if (e >= 0 && e < p.n_pages) atomicOr(&p.live[e >> 5], 1u << (e & 31));
      else record_status(p.hdr, XKV_ERR_INVALID_ARG);
    }
  }
  phase();
  const int n_words = (p.n_pages + 31) / 32;
  int64_t word0, word1;
  cta_run(n_words, &word0, &word1);
  int mine = 0;
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    int total;
    block_scan(w < word1 ? __popc(__ldcg(&p.live[w])) : 0, s_scan, &total);
    mine += total;
  }
  if (threadIdx.x == 0) p.counts[blockIdx.x] = mine;
  phase();
  int n_live = 0;
  for (int i = 0; i < (int)gridDim.x; ++i) n_live += __ldcg(&p.counts[i]);
  // bits of word w below and from n_live on
  auto below = [&](int64_t w) -> uint32_t {
    const int64_t at = (int64_t)n_live - w * 32;
    return at >= 32 ? 0xffffffffu : (at <= 0 ? 0u : (1u << at) - 1u);
  };
  int gaps = 0, moved = 0;
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    const uint32_t bits = w < word1 ? __ldcg(&p.live[w]) : 0u, low = w < word1 ? below(w) : 0u;
    int t0, t1;
    block_scan(__popc(~bits & low), s_scan, &t0);
    block_scan(__popc(bits & ~low), s_scan, &t1);
    gaps += t0;
    moved += t1;
  }
  if (threadIdx.x == 0) {
    p.counts[kMaxCluster + blockIdx.x] = gaps;
    p.counts[2 * kMaxCluster + blockIdx.x] = moved;
  }
  phase();
  gaps = moved = 0;
  for (int i = 0; i < (int)blockIdx.x; ++i) {
    gaps += __ldcg(&p.counts[kMaxCluster + i]);
    moved += __ldcg(&p.counts[2 * kMaxCluster + i]);
  }
  for (int64_t base = word0; base < word1; base += kPlanThreads) {
    const int64_t w = base + threadIdx.x;
    const uint32_t bits = w < word1 ? __ldcg(&p.live[w]) : 0u, low = w < word1 ? below(w) : 0u;
    int t0, t1;
    int gap = gaps + block_scan(__popc(~bits & low), s_scan, &t0), go = moved + block_scan(__popc(bits & ~low), s_scan, &t1);
    gaps += t0;
    moved += t1;
    if (w < word1) {
      p.live[w] = 0u;
      const int n = (int)min((int64_t)32, p.n_pages - w * 32);
      for (int i = 0; i < n; ++i) {
        const int page = (int)w * 32 + i;
        const bool in_use = (bits >> i) & 1u, in_front = (low >> i) & 1u;
        if (in_front) {
          if (!in_use) p.list[gap++].dst = page;
          else if (p.shares != nullptr) p.shares[page] = p.shares_before[page];
        } else if (in_use) {
          p.list[go].src = page;
          p.list[go].rows = p.page_size;
          p.place[page] = go++;
        } else if (p.shares != nullptr) {
          p.shares[page] = 0;
        }
      }
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int all = 0;
    for (int i = 0; i < (int)gridDim.x; ++i) all += __ldcg(&p.counts[2 * kMaxCluster + i]);
    *p.n_live = n_live;
    *p.n_moved = all;
    *p.used = n_live;
  }
}

// Tables, counters of the pages that move, the list; then the pages.
__global__ void __launch_bounds__(kCopyThreads) compact_move_kernel(const CompactParams p, const CopyParams c) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int n_live = __ldcg(p.n_live), n_moved = __ldcg(p.n_moved);
  const int64_t tid = (int64_t)blockIdx.x * kCopyThreads + threadIdx.x, step = (int64_t)gridDim.x * kCopyThreads;
  const int64_t n_entries = (int64_t)p.n_layers * p.batch * p.cols;
  for (int64_t i = tid; i < n_entries; i += step) {
    const int64_t row = i / p.cols;
    const int e = p.before[i];
    int now = e;
    if (e >= n_live && e < p.n_pages) {
      const int have = (min(max(__ldg(&p.lens[row]), 0), p.cols * p.page_size) + p.page_size - 1) / p.page_size;
      if (i - row * p.cols < have) now = __ldcg(&p.list[__ldcg(&p.place[e])].dst);
    }
    p.table[i] = now;
  }
  if (p.free_pages != nullptr)
    for (int64_t i = n_live + tid; i < p.n_pages; i += step) p.free_pages[i] = (int)i;
  if (p.shares != nullptr)
    for (int64_t i = tid; i < n_moved; i += step) {
      const int src = __ldcg(&p.list[i].src), held = p.shares_before[src];
      p.shares[src] = 0;
      p.shares[__ldcg(&p.list[i].dst)] = held;
    }
  const int64_t per = 2 * (int64_t)c.n_kv_heads * c.pieces, n = n_moved * per;
  for (int64_t u = tid >> 5; u < n; u += step >> 5) {
    const RowCopy x = {__ldcg(&p.list[u / per].src), __ldcg(&p.list[u / per].dst), c.page_size};
    copy_piece(c, x, (int)(u % per));
  }
}

// ---------------------------------------------------------------------------------------------
// Host side
// ---------------------------------------------------------------------------------------------
struct Layout {
  size_t counts, list, a, b, bits, fresh, total;
};

Layout fork_layout(int64_t n_rows, int cols, int64_t n_pages) {
  Layout L;
  size_t off = kHeaderBytes;
  L.counts = off; off = align_up(off + (8 + 2 * kMaxCluster) * 4, 256);
  L.bits = off;   off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.list = off;   off = align_up(off + (size_t)n_rows * sizeof(RowCopy), 256);
  L.a = off;      off = align_up(off + (size_t)n_rows * 4, 256);
  L.b = off;      off = align_up(off + (size_t)n_rows * 4, 256);
  L.fresh = off;  off = align_up(off + (size_t)n_rows * cols * 4, 256);
  L.total = off;
  return L;
}

Layout compact_layout(int64_t n_pages) {
  Layout L = {};
  size_t off = kHeaderBytes;
  L.counts = off; off = align_up(off + (8 + 3 * kMaxCluster) * 4, 256);
  L.bits = off;   off = align_up(off + (size_t)(n_pages + 31) / 32 * 4, 256);
  L.list = off;   off = align_up(off + (size_t)n_pages * sizeof(RowCopy), 256);
  L.a = off;      off = align_up(off + (size_t)n_pages * 4, 256);
  L.total = off;
  return L;
}

template <typename P>
xkv_status launch_cluster(void (*kernel)(P), const P& p, int ctas, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(kPlanThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = (unsigned)ctas;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) {
    (void)cudaGetLastError();
    return XKV_ERR_CUDA;
  }
  count_launch();
  return check_launch();
}

template <typename... Args>
xkv_status launch_after(void (*kernel)(Args...), int grid, cudaStream_t st, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)grid);
  cfg.blockDim = dim3(kCopyThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr;           // its CTAs are in place when the plan ends
  attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr.val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = &attr;
  cfg.numAttrs = 1;
  if (cudaLaunchKernelEx(&cfg, kernel, args...) != cudaSuccess) {
    (void)cudaGetLastError();
    return XKV_ERR_CUDA;
  }
  count_launch();
  return check_launch();
}

// CTAs of a plan: one (whose barriers are cheapest) for a few hundred caches of short tables, else a cluster.
int plan_ctas(int64_t n_rows, int cols) { return n_rows * ((cols + 31) / 32) <= 2 * kPlanWarps ? 1 : kMaxCluster; }

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
  p.n_layers = c->n_layers;
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
  p.gone = reinterpret_cast<uint32_t*>(ws + L.bits);
  p.fresh = reinterpret_cast<int32_t*>(ws + L.fresh);
  xkv_status s = launch_cluster(fork_kernel, p, plan_ctas(n_rows, p.cols), st);
  if (s != XKV_OK) return s;
  const CopyParams cp = copy_params(d, c, c);
  return launch_after(copy_rows_kernel, copy_grid(cp, n_rows), st, cp, (const RowCopy*)p.list, (const int32_t*)p.n_copies);
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
  p.n_layers = c->n_layers;
  p.batch = d->batch;
  p.cols = c->max_pages_per_seq;
  p.page_size = c->page_size;
  p.n_pages = c->n_pages;
  p.hdr = reinterpret_cast<WorkspaceHeader*>(ws);
  p.n_live = reinterpret_cast<int32_t*>(ws + L.counts);
  p.n_moved = p.n_live + 1;
  p.counts = p.n_live + 8;
  p.live = reinterpret_cast<uint32_t*>(ws + L.bits);
  p.list = reinterpret_cast<RowCopy*>(ws + L.list);
  p.place = reinterpret_cast<int32_t*>(ws + L.a);
  xkv_status s = launch_cluster(compact_kernel, p, plan_ctas(n_rows, p.cols), st);
  if (s != XKV_OK) return s;
  const CopyParams cp = copy_params(d, c, c);
  const int64_t entries = (n_rows * p.cols + 31) / 32;
  const int grid = std::max(copy_grid(cp, std::min<int64_t>(c->n_pages, n_rows * p.cols)),
                            (int)std::min<int64_t>(entries / (kCopyThreads / 32), sm_count()));
  return launch_after(compact_move_kernel, grid, st, p, cp);
}

xkv_status copy_pages(const xkv_dims* d, const xkv_cache* from, const int32_t* src, const xkv_cache* to, const int32_t* dst,
                      int64_t n_copies, void* workspace, cudaStream_t st) {
  const CopyParams p = copy_params(d, from, to);
  copy_pages_kernel<<<copy_grid(p, n_copies), kCopyThreads, 0, st>>>(p, src, dst, n_copies, from->n_pages, to->n_pages,
                                                                     static_cast<WorkspaceHeader*>(workspace));
  count_launch();
  return check_launch();
}

}  // namespace xkv
